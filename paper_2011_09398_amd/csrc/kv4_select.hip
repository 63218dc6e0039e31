// Choosing pages of the 4-bit cache by the signs of queries and keys.
#include "kv4_attend.hpp"

namespace lce {
namespace kv4 {
namespace {

constexpr int kWaves = kThreads / 64;

// Ranks are 16 bits: 0 = not to be chosen, else 1 + (group*D - d) for the
// smallest number d of differing sign bits over the page's visible tokens (the
// score is group*D - 2d), 65535 for a page that is kept in any case.
constexpr uint32_t kKept = 65535;

// Pages whose ranks are kept in LDS while the best are looked for; those of
// longer sequences are read from the workspace.
constexpr int kHeld = 4096;

// The largest over a wave, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    const auto step = [&](uint32_t w) { v = max(v, w); };
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));    // quads
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));   // half rows
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));   // rows
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

// Exclusive prefix sum of one value per thread; every thread gets the total.
__device__ __forceinline__ int scan(int v, int *sums, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    __syncthreads();
    return before + x - v;
}

// The digit value d at which the count of ranks with larger digits first leaves
// fewer than `want`: on return `want` is what is still to be taken at d itself.
// One histogram bin per thread.
__device__ __forceinline__ int pick_digit(const int *bins, int *sums, int *result, int &want) {
    const int d = kThreads - 1 - (int)threadIdx.x;   // thread 0 has the largest digit
    const int mine = bins[d];
    int total;
    const int above = scan(mine, sums, total);
    if (above < want && above + mine >= want) {
        result[0] = d;
        result[1] = want - above;
    }
    __syncthreads();
    want = result[1];
    const int found = result[0];
    __syncthreads();
    return found;
}

// Writes the chosen pages of one token and head: the ranks of all its pages ->
// the best p.list of them, in order.
__device__ __forceinline__ void choose(const uint16_t *ranks, int pages, const SelectParams &p,
                                       int *bins, int *sums, int *result) {
    // the rank of the last page taken, digit by digit, and how many pages of that
    // very rank are taken
    int have = 0;
    for (int i = threadIdx.x; i < pages; i += kThreads) have += ranks[i] != 0;
    int total;
    scan(have, sums, total);
    const int count = min(p.list, total);
    uint32_t least = 1;
    int equal = count;
    if (total > p.list) {
        int want = count;
        bins[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < pages; i += kThreads) atomicAdd(&bins[ranks[i] >> 8], 1);
        __syncthreads();
        const int high = pick_digit(bins, sums, result, want);
        bins[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < pages; i += kThreads)
            if (ranks[i] >> 8 == high) atomicAdd(&bins[ranks[i] & 255], 1);
        __syncthreads();
        least = (uint32_t)(high << 8 | pick_digit(bins, sums, result, want));
        equal = want;
    } else {
        equal = 0;   // all with a rank: none is held back
        least = 0;
    }

    // each thread has a run of pages; of those with rank `least` the first
    // `equal` are taken
    int32_t *out = p.chosen + (int64_t)blockIdx.x * p.list;
    const int run = (pages + kThreads - 1) / kThreads;
    const int from = min((int)threadIdx.x * run, pages), to = min(from + run, pages);
    int more = 0, same = 0;
    for (int i = from; i < to; ++i) {
        more += ranks[i] > least;
        same += ranks[i] == least;
    }
    int at = scan(more, sums, total), ties = scan(same, sums, total);
    for (int i = from; i < to; ++i) {
        const uint32_t r = ranks[i];
        if (r > least) {
            out[at + min(ties, equal)] = i;
            ++at;
        } else if (r == least) {
            if (ties < equal) out[at + ties] = i;
            ++ties;
        }
    }
    for (int i = count + threadIdx.x; i < p.list; i += kThreads) out[i] = -1;
}

}  // namespace

// Grid (tokens * kv_heads, splits), four waves.  A wave takes four pages at a
// time, a lane a token of each: the token's signs, 16 bytes for 128 channels,
// against the packed signs of the query heads, which are the same for all lanes.
// The last split of a token and head to finish chooses: the rank of the last
// page taken comes from two histograms of 8 bits, and a prefix sum puts the
// chosen pages in order.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void select_kernel(SelectParams p) {
    constexpr int W = D / 32, U = 4;
    __shared__ int bins[256];
    __shared__ int sums[kWaves];
    __shared__ int result[2];
    __shared__ int last;
    __shared__ uint16_t held[kHeld];
    extern __shared__ u32x2 signs[];   // [group][W / 2]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % p.kv_heads, token = blockIdx.x / p.kv_heads;
    const int split = blockIdx.y;
    const T *q = (const T *)p.q + (int64_t)token * p.q_token + (int64_t)head * p.group * p.q_head;
    // the query heads' signs: a ballot packs 64 channels
    for (int h = wave; h < p.group; h += kWaves)
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            const uint64_t b =
                __builtin_amdgcn_ballot_w64((float)q[h * p.q_head + 64 * c + lane] < 0.0f);
            if (lane == 0) signs[h * (W / 2) + c] = u32x2{(uint32_t)b, (uint32_t)(b >> 32)};
        }
    const Sequence seq = find_sequence(p.q_start, p.lengths, p.seqs, p.tokens, p.width, token,
                                       [](int s, int) { return (int64_t)s; });
    if (seq.index < 0 || token - seq.start >= seq.queries) return;
    const Span span = visible(seq, token - seq.start, p.causal, p.window);
    const int pages = (span.hi + kPage - 1) / kPage;
    const int splits = clampi((pages + p.chunk - 1) / p.chunk, 1, (int)gridDim.y);
    if (split >= splits) return;
    const int begin = split * p.chunk, end = split == splits - 1 ? pages : begin + p.chunk;
    __syncthreads();

    const int32_t *table = p.table + (int64_t)seq.index * p.width;
    const uint8_t *cache = p.cache + (int64_t)head * Record<D>::kBytes + Record<D>::kSigns;
    const int64_t stride = (int64_t)p.kv_heads * Record<D>::kBytes;
    uint16_t *ranks = p.ranks + (int64_t)blockIdx.x * p.width;
    const uint32_t top = p.group * D + 1;
    // a wave's pages are runs of U, kWaves * U apart; the table's entries of 64 / U
    // such runs at a time, one a lane
    for (int run = begin + wave * U; run < end; run += kWaves * 64) {
        const int mine = run + lane / U * (kWaves * U) + lane % U;
        int phys = mine < end ? table[mine] : -1;
        if (phys >= p.pages || (mine + 1) * (int64_t)kPage <= span.lo) phys = -1;
        uint32_t kept = 0;   // lane i: the rank of this lane's page
        for (int i = 0; i < 64 && run + i / U * (kWaves * U) < end; i += U) {
            u32x2 k[U][W / 2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t at = max(__builtin_amdgcn_readlane(phys, i + u), 0);
                const u32x2 *from =
                    reinterpret_cast<const u32x2 *>(cache + at * stride + lane * (D / 8));
#pragma unroll
                for (int w = 0; w < W / 2; ++w) k[u][w] = from[w];
            }
            uint32_t d[U] = {0, 0, 0, 0};
            for (int h = 0; h < p.group; ++h)
#pragma unroll
                for (int w = 0; w < W / 2; ++w) {
                    const u32x2 s = signs[h * (W / 2) + w];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        d[u] += __builtin_popcount(k[u][w][0] ^ s[0]);
                        d[u] += __builtin_popcount(k[u][w][1] ^ s[1]);
                    }
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int page = run + i / U * (kWaves * U) + u;
                const int j = page * kPage + lane;
                uint32_t rank = j >= span.lo && j < span.hi ? top - d[u] : 0;
                rank = wave_max(rank);
                kept = lane == i + u ? rank : kept;
            }
        }
        if (mine < end) {
            if (phys < 0) kept = 0;
            if (kept && (mine < p.keep_first || mine >= pages - p.keep_last)) kept = kKept;
            if (splits > 1 || pages > kHeld)
                __hip_atomic_store(ranks + mine, (uint16_t)kept, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
            else
                held[mine] = (uint16_t)kept;
        }
    }

    if (splits > 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) last = last_of(p.tickets + (int64_t)blockIdx.x * kTicketStride, splits);
        __syncthreads();
        if (!last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        if (pages <= kHeld)
            for (int i = threadIdx.x; i < pages; i += kThreads) held[i] = ranks[i];
    }
    __syncthreads();
    if (pages <= kHeld)
        choose(held, pages, p, bins, sums, result);
    else
        choose(ranks, pages, p, bins, sums, result);
}

namespace {

template <typename T>
void launch_t(const SelectParams &p, int dim, dim3 grid, hipStream_t s) {
    const size_t lds = (size_t)p.group * (dim / 8);
    if (dim == 64)
        hipLaunchKernelGGL((select_kernel<T, 64>), grid, dim3(kThreads), lds, s, p);
    else if (dim == 128)
        hipLaunchKernelGGL((select_kernel<T, 128>), grid, dim3(kThreads), lds, s, p);
    else
        hipLaunchKernelGGL((select_kernel<T, 256>), grid, dim3(kThreads), lds, s, p);
}

}  // namespace

void launch_select(const SelectParams &p, int type, int dim, dim3 grid, hipStream_t s) {
    if (type == LCE_FLOAT16) launch_t<_Float16>(p, dim, grid, s);
    else launch_t<__bf16>(p, dim, grid, s);
}

}  // namespace kv4
}  // namespace lce
