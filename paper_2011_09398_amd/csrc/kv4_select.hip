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

}  // namespace

// Grid (tokens * kv_heads, splits), four waves.  A wave takes a page at a time,
// a lane a token: the token's signs, 16 bytes for 128 channels, against the
// packed signs of the query heads, which are the same for all lanes.  The last
// split of a token and head to finish chooses: the rank of the last page taken
// comes from two histograms of 8 bits, and a prefix sum puts the chosen pages in
// order.
// Bound by memory for up to about 8 query heads a cache head, by XOR and
// population count (two operations per 32 channels, head and token) for more.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void select_kernel(SelectParams p) {
    constexpr int W = D / 32;
    __shared__ int bins[256];
    __shared__ int sums[kWaves];
    __shared__ int result[2];
    __shared__ int last;
    extern __shared__ uint32_t signs[];   // [group][W]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % p.kv_heads, token = blockIdx.x / p.kv_heads;
    const int split = blockIdx.y;
    const Sequence seq = find_sequence(p.q_start, p.lengths, p.seqs, p.tokens, p.width, token,
                                       [](int s, int) { return (int64_t)s; });
    if (seq.index < 0 || token - seq.start >= seq.queries) return;
    const Span span = visible(seq, token - seq.start, p.causal, p.window);
    const int pages = (span.hi + kPage - 1) / kPage;
    const int splits = clampi((pages + p.chunk - 1) / p.chunk, 1, (int)gridDim.y);
    if (split >= splits) return;
    const int begin = split * p.chunk, end = split == splits - 1 ? pages : begin + p.chunk;

    // the query heads' signs: a ballot packs 64 channels
    const T *q = (const T *)p.q + (int64_t)token * p.q_token + (int64_t)head * p.group * p.q_head;
    for (int h = wave; h < p.group; h += kWaves)
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            const uint64_t b =
                __builtin_amdgcn_ballot_w64((float)q[h * p.q_head + 64 * c + lane] < 0.0f);
            if (lane == 0) {
                signs[h * W + 2 * c] = (uint32_t)b;
                signs[h * W + 2 * c + 1] = (uint32_t)(b >> 32);
            }
        }
    __syncthreads();

    const int32_t *table = p.table + (int64_t)seq.index * p.width;
    const uint8_t *cache = p.cache + (int64_t)head * Record<D>::kBytes + Record<D>::kSigns;
    uint16_t *ranks = p.ranks + (int64_t)blockIdx.x * p.width;
    const int top = p.group * D + 1;
    for (int page = begin + wave; page < end; page += kWaves) {
        const int phys = __builtin_amdgcn_readfirstlane(table[page]);
        uint32_t rank = 0;
        if (phys >= 0 && phys < p.pages && (page + 1) * kPage > span.lo) {
            const uint32_t *at = reinterpret_cast<const uint32_t *>(
                cache + (int64_t)phys * p.kv_heads * Record<D>::kBytes + lane * (D / 8));
            uint32_t k[W];
#pragma unroll
            for (int w = 0; w < W; w += 2) {
                const u32x2 x = *reinterpret_cast<const u32x2 *>(at + w);
                k[w] = x[0], k[w + 1] = x[1];
            }
            uint32_t d = 0;
            for (int h = 0; h < p.group; ++h)
#pragma unroll
                for (int w = 0; w < W; ++w) d += __builtin_popcount(k[w] ^ signs[h * W + w]);
            const int j = page * kPage + lane;
            rank = j >= span.lo && j < span.hi ? (uint32_t)top - d : 0;
#pragma unroll
            for (int s = 1; s < 64; s *= 2) rank = max(rank, (uint32_t)__shfl_xor((int)rank, s));
            if (rank && (page < p.keep_first || page >= pages - p.keep_last)) rank = kKept;
        }
        if (lane == 0)
            __hip_atomic_store(ranks + page, (uint16_t)rank, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    }

    if (splits > 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) last = last_of(p.tickets + (int64_t)blockIdx.x * kTicketStride, splits);
        __syncthreads();
        if (!last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    } else {
        __syncthreads();
    }

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
