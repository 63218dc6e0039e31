// Choosing pages of the 4-bit cache by the signs of queries and keys.
#include <type_traits>

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

// Bits of the number of query heads of a cache head: at most 65280 / 64.
constexpr int kPlanes = 10;
constexpr int kInRegisters = 4;

// The largest over a wave of each of four values: lane l gets that of v[l % 4].
// The first two exchanges leave two values, then one, in each lane.
__device__ __forceinline__ uint32_t wave_max4(const uint32_t (&v)[4]) {
    const int lane = threadIdx.x & 63;
    const auto quad = [](uint32_t x, auto ctrl) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF,
                                                     true);
    };
    const bool odd = lane & 1, upper = lane & 2;
    const std::integral_constant<int, 0xB1> by1;     // quad_perm: lane ^ 1
    const std::integral_constant<int, 0x4E> by2;     // quad_perm: lane ^ 2
    const std::integral_constant<int, 0x124> by4;    // row_ror: 4 lanes on
    const std::integral_constant<int, 0x128> by8;    // row_ror: 8 lanes on
    const uint32_t a = max(odd ? v[1] : v[0], quad(odd ? v[0] : v[1], by1));
    const uint32_t b = max(odd ? v[3] : v[2], quad(odd ? v[2] : v[3], by1));
    uint32_t x = max(upper ? b : a, quad(upper ? a : b, by2));
    x = max(x, quad(x, by4));
    x = max(x, quad(x, by8));
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((uint32_t)r[0], (uint32_t)r[1]);
    const auto s = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max((uint32_t)s[0], (uint32_t)s[1]);
}

// Pages of a rank's upper and lower eight bits.
struct Bins {
    int high[256], low[256];
};

// The digit at which the pages with larger digits first leave fewer than `want`:
// on return `want` is what is still to be taken at that digit.  Every wave finds
// it for itself, four digits a lane, the largest in lane 0.
__device__ __forceinline__ int pick_digit(const int *bins, int &want) {
    const int lane = threadIdx.x & 63;
    int n[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        n[i] = bins[255 - 4 * lane - i];
        mine += n[i];
    }
    int above = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(above, d);
        if (lane >= d) above += y;
    }
    above -= mine;
    int digit = -1, left = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (digit < 0 && above + n[i] >= want) {
            digit = 255 - 4 * lane - i;
            left = want - above;
        }
        above += n[i];
    }
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(digit >= 0));
    want = __builtin_amdgcn_readlane(left, at);
    return __builtin_amdgcn_readlane(digit, at);
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                     __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Writes the chosen pages of one token and head: the ranks of all its pages ->
// the best p.list of them, in order.  `bins` are zero.
__device__ __forceinline__ void choose(const uint16_t *ranks, int pages, const SelectParams &p,
                                       Bins &bins, int (&counts)[kWaves][2]) {
    // the rank of the last page taken, digit by digit, and how many pages of that
    // very rank are taken: the first ones
    uint32_t least = 0;
    int equal = 0;
    if (pages > p.list) {
        int want = p.list;
        for (int i = threadIdx.x; i < pages; i += kThreads) atomicAdd(&bins.high[ranks[i] >> 8], 1);
        __syncthreads();
        const int high = pick_digit(bins.high, want);
        for (int i = threadIdx.x; i < pages; i += kThreads)
            if (ranks[i] >> 8 == high) atomicAdd(&bins.low[ranks[i] & 255], 1);
        __syncthreads();
        least = (uint32_t)(high << 8 | pick_digit(bins.low, want));
        equal = least ? want : 0;   // rank 0 is never taken
    }
    // a run of pages for each wave: what it takes, what the waves before it take,
    // and then each page's place
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int run = (pages + kThreads - 1) / kThreads * 64;
    const int from = wave * run, to = min(from + run, pages);
    int more = 0, same = 0;
    for (int i = from; i < to; i += 64) {
        const uint32_t r = i + lane < to ? ranks[i + lane] : 0;
        more += __builtin_popcountll(__builtin_amdgcn_ballot_w64(r > least));
        same += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < to && r == least));
    }
    if (lane == 0) counts[wave][0] = more, counts[wave][1] = same;
    __syncthreads();
    int at = 0, ties = 0, all = 0, all_ties = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) at = all, ties = all_ties;
        all += counts[w][0];
        all_ties += counts[w][1];
    }
    int32_t *out = p.chosen + (int64_t)blockIdx.x * p.list;
    for (int i = from; i < to; i += 64) {
        const uint32_t r = i + lane < to ? ranks[i + lane] : 0;
        const uint64_t above = __builtin_amdgcn_ballot_w64(r > least);
        const uint64_t level = __builtin_amdgcn_ballot_w64(i + lane < to && r == least);
        const int tie = ties + lanes_below(level);
        const int place = at + lanes_below(above) + min(tie, equal);
        if (r > least || (i + lane < to && r == least && tie < equal)) out[place] = i + lane;
        at += __builtin_popcountll(above);
        ties += __builtin_popcountll(level);
    }
    for (int i = all + min(all_ties, equal) + threadIdx.x; i < p.list; i += kThreads) out[i] = -1;
}

}  // namespace

// Grid (tokens * kv_heads, splits), four waves.  A wave takes four pages at a
// time, a lane a token of each: the token's signs, 16 bytes for 128 channels,
// against the packed signs of the query heads, which are the same for all lanes.
// The last split of a token and head to finish chooses: the rank of the last
// page taken comes from two histograms of 8 bits, and a prefix sum puts the
// chosen pages in order.
//
// Bound by memory where contexts are long: 32 sequences of up to 32768 tokens, 64 heads
// of 128 on 8 (50 MB of signs) take 22.1 us, of which the scores take 10 (5 TB/s), the
// ticket and the choice 3.7, and the launch and all before the first page the rest.
// Small calls wait for the host: 8 sequences of up to 8192 tokens, 32 heads on 8, 7.6 us.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void select_kernel(SelectParams p) {
    constexpr int W = D / 32, U = 4;
    __shared__ Bins bins;
    __shared__ int counts[kWaves][2];
    __shared__ int negatives[W];
    __shared__ int last;
    __shared__ uint16_t held[kHeld];
    extern __shared__ uint32_t signs[];   // [group][W], then the planes [kPlanes][W]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % p.kv_heads, token = blockIdx.x / p.kv_heads;
    const int split = blockIdx.y;
    // eight channels of a query head a thread
    const T *q = (const T *)p.q + (int64_t)token * p.q_token + (int64_t)head * p.group * p.q_head;
    const int eights = p.group * (D / 8);
    u32x4 x = {0, 0, 0, 0};
    if ((int)threadIdx.x < eights)
        x = *reinterpret_cast<const u32x4 *>(q + threadIdx.x / (D / 8) * p.q_head +
                                             threadIdx.x % (D / 8) * 8);
    bins.high[threadIdx.x] = bins.low[threadIdx.x] = 0;
    const Sequence seq = find_sequence(p.q_start, p.lengths, p.seqs, p.tokens, p.width, token,
                                       [](int s, int) { return (int64_t)s; });
    if (seq.index < 0 || token - seq.start >= seq.queries) return;
    const Span span = visible(seq, token - seq.start, p.causal, p.window);
    const int pages = (span.hi + kPage - 1) / kPage;
    // as many splits as the grid has, of whole runs of all waves; at least p.chunk pages
    const int least = (pages + (int)gridDim.y - 1) / (int)gridDim.y;
    const int chunk = max(p.chunk, (least + kWaves * U - 1) / (kWaves * U) * (kWaves * U));
    const int splits = max((pages + chunk - 1) / chunk, 1);
    if (split >= splits) return;
    const int begin = split * chunk, end = min(begin + chunk, pages);

    for (int e = threadIdx.x; e < eights; e += kThreads) {
        if (e >= kThreads)
            x = *reinterpret_cast<const u32x4 *>(q + e / (D / 8) * p.q_head + e % (D / 8) * 8);
        uint32_t b = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            b |= ((float)bits_as<T>((uint16_t)(x[i / 2] >> (i % 2 * 16))) < 0.0f ? 1u : 0u) << i;
        reinterpret_cast<uint8_t *>(signs)[e] = (uint8_t)b;
    }
    // With n_c the number of heads whose channel c is negative and k_c the key's
    // sign bit, the differing bits over all heads are
    //     sum_c n_c + group * sum_c k_c - 2 sum_c k_c n_c,
    // and the last sum goes by the bits of n_c: plane i holds bit i of every n_c.
    // Two operations a plane instead of a head: 5 planes for 16 heads.
    const int planes = 32 - __builtin_clz(p.group);
    uint32_t *plane = signs + p.group * W;
    __syncthreads();
    if (threadIdx.x < W) {
        uint32_t n[kPlanes] = {};
        for (int h = 0; h < p.group; ++h) {
            uint32_t carry = signs[h * W + threadIdx.x];
#pragma unroll
            for (int i = 0; i < kPlanes; ++i)
                if (i < planes) {
                    const uint32_t sum = n[i] ^ carry;
                    carry &= n[i];
                    n[i] = sum;
                }
        }
        uint32_t all = 0;
#pragma unroll
        for (int i = 0; i < kPlanes; ++i) {
            plane[i * W + threadIdx.x] = n[i];
            all += (uint32_t)__builtin_popcount(n[i]) << i;
        }
        negatives[threadIdx.x] = (int)all;
    }
    __syncthreads();
    uint32_t top = p.group * D + 1;   // rank of a key that agrees in every bit
#pragma unroll
    for (int w = 0; w < W; ++w) top -= negatives[w];
    // the first planes stay in scalar registers; more than 15 heads need others
    uint32_t mask[kInRegisters][W];
#pragma unroll
    for (int j = 0; j < kInRegisters; ++j)
#pragma unroll
        for (int w = 0; w < W; ++w)
            mask[j][w] = __builtin_amdgcn_readfirstlane(plane[j * W + w]);

    const int32_t *table = p.table + (int64_t)seq.index * p.width;
    const uint8_t *cache = p.cache + (int64_t)head * Record<D>::kBytes + Record<D>::kSigns;
    const int64_t stride = (int64_t)p.kv_heads * Record<D>::kBytes;
    uint16_t *ranks = p.ranks + (int64_t)blockIdx.x * p.width;
    // a wave's pages are runs of U, kWaves * U apart; the table's entries of 64 / U
    // such runs at a time, one a lane
    for (int run = begin + wave * U; run < end; run += kWaves * 64) {
        const int mine = run + lane / U * (kWaves * U) + lane % U;
        int phys = mine < end ? table[mine] : -1;
        if (phys >= p.pages || (mine + 1) * (int64_t)kPage <= span.lo) phys = -1;
        uint32_t kept = 0;   // lane i: the rank of this lane's page
        uint32_t k[U][W];
        const auto load = [&](int i) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t at = max(__builtin_amdgcn_readlane(phys, i + u), 0);
                const u32x2 *from =
                    reinterpret_cast<const u32x2 *>(cache + at * stride + lane * (D / 8));
#pragma unroll
                for (int w = 0; w < W; w += 2) {
                    const u32x2 y = from[w / 2];
                    k[u][w] = y[0], k[u][w + 1] = y[1];
                }
            }
        };
        load(0);
        for (int i = 0; i < 64 && run + i / U * (kWaves * U) < end; i += U) {
            uint32_t bits[U], agree[U];
            uint32_t now[U][W];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int w = 0; w < W; ++w) now[u][w] = k[u][w];
            if (i + U < 64 && run + (i / U + 1) * (kWaves * U) < end) load(i + U);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                bits[u] = agree[u] = 0;
#pragma unroll
                for (int w = 0; w < W; ++w) bits[u] += __builtin_popcount(now[u][w]);
            }
            const auto add = [&](int u, const uint32_t (&m)[W]) {
                agree[u] *= 2;
#pragma unroll
                for (int w = 0; w < W; ++w) agree[u] += __builtin_popcount(now[u][w] & m[w]);
            };
            for (int j = planes - 1; j >= kInRegisters; --j) {
                uint32_t m[W];
#pragma unroll
                for (int w = 0; w < W; ++w) m[w] = plane[j * W + w];
#pragma unroll
                for (int u = 0; u < U; ++u) add(u, m);
            }
#pragma unroll
            for (int j = kInRegisters - 1; j >= 0; --j)
                if (j < planes) {
#pragma unroll
                    for (int u = 0; u < U; ++u) add(u, mask[j]);
                }
            const int page = run + i / U * (kWaves * U);
            uint32_t rank[U];
#pragma unroll
            for (int u = 0; u < U; ++u) rank[u] = top + 2 * agree[u] - (uint32_t)p.group * bits[u];
            if (page * kPage < span.lo || (page + U) * kPage > span.hi) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int j = (page + u) * kPage + lane;
                    rank[u] = j >= span.lo && j < span.hi ? rank[u] : 0;
                }
            }
            const uint32_t best = wave_max4(rank);   // lane l: of page l % U
            kept = lane / U == i / U ? best : kept;
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
        if (pages <= kHeld)
            for (int i = threadIdx.x; i < pages; i += kThreads)
                held[i] = __hip_atomic_load(ranks + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        else
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    }
    __syncthreads();
    if (pages <= kHeld)
        choose(held, pages, p, bins, counts);
    else
        choose(ranks, pages, p, bins, counts);
}

namespace {

template <typename T>
void launch_t(const SelectParams &p, int dim, dim3 grid, hipStream_t s) {
    const size_t lds = (size_t)(p.group + kPlanes) * (dim / 8);
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
