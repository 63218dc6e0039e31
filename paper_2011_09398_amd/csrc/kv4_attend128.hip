// Attention over the 4-bit cache, 128 query rows a tile: prompts.
#include "kv4_attend.hpp"

namespace lce {
namespace kv4 {
namespace {

constexpr int kWaves = kThreads / 64;
constexpr int kWaveRows = 32;
constexpr int kRows = kWaves * kWaveRows;

// The keys of a page as first operands of 32x32x64 products: lane (n, h), n =
// lane % 32, h = lane / 32, holds of tokens n and 32 + n the 32 channels from
// 64c + 32h on.
template <int D>
struct Keys {
    static constexpr int kChunks = D / 64;
    u32x4 k[2][kChunks];
    uint32_t scale[kChunks];   // byte 2t + n / 16: scale of token 32t + n

    __device__ __forceinline__ void load(const uint8_t *rec, int n, int h) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
                k[t][c] = *reinterpret_cast<const u32x4 *>(rec + (32 * t + n) * (D / 2) + 32 * c +
                                                           16 * h);
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            scale[c] = *reinterpret_cast<const uint32_t *>(rec + Record<D>::kKeyScale +
                                                           (n % 16 * (D / 32) + 2 * c + h) * 4);
    }
};

// One wave's quarter of a page's values, 16 tokens: lane (r, g), r = lane % 16, g =
// lane / 16, holds tokens 4g .. 4g + 3 of the D/16 channels from D/16 * r on.
template <int D>
struct Values {
    uint32_t v[D / 32];
    uint32_t scale;   // byte i: token 4g + i

    __device__ __forceinline__ void load(const uint8_t *rec, int quarter, int r, int g) {
        const uint8_t *at = rec + Record<D>::kValue + ((4 * quarter + g) * 16 + r) * (D / 8);
        if constexpr (D == 64) {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(at);
            v[0] = w[0], v[1] = w[1];
        } else {
#pragma unroll
            for (int j = 0; j < D / 128; ++j) {
                const u32x4 w = reinterpret_cast<const u32x4 *>(at)[j];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * j + i] = w[i];
            }
        }
        scale = *reinterpret_cast<const uint32_t *>(rec + Record<D>::kValueScale +
                                                    (r * D / 512) * 64 + 16 * g + 4 * quarter);
    }
};

// A page's values in LDS, two bytes each, in the order in which the product with
// the weights reads them: for 16 tokens at a time and each half of the wave, 16
// bytes for each channel, of tokens 4h .. 4h + 3 and 8 + 4h .. 8 + 4h + 3 (those
// whose scores the half has); channel D/16 * r + m at place 16m + r, so that a
// wave writes and reads runs of memory.
template <int D>
struct Page {
    u32x4 unit[4][2][D];
};

template <typename E, int D, int B, bool SAT = false>
__device__ __forceinline__ void store_values(Page<D> &page, const Values<D> &x, int quarter, int r,
                                             int g) {
    if constexpr (B < D / 32) {
        constexpr int G = D / 32;   // bytes of a token
        const uint32_t w = x.scale;
        const uint32_t x0 = decode_pair<E, B % 4, SAT>(x.v[B / 4], bits_as<float>(w << 23));
        const uint32_t x1 =
            decode_pair<E, (G + B) % 4, SAT>(x.v[(G + B) / 4], bits_as<float>(w << 15));
        const uint32_t x2 =
            decode_pair<E, (2 * G + B) % 4, SAT>(x.v[(2 * G + B) / 4], bits_as<float>(w << 7));
        const uint32_t x3 =
            decode_pair<E, (3 * G + B) % 4, SAT>(x.v[(3 * G + B) / 4], bits_as<float>(w >> 1));
        // two tokens of a channel side by side
        const u32x2 even = {__builtin_amdgcn_perm(x1, x0, 0x05040100u),
                            __builtin_amdgcn_perm(x3, x2, 0x05040100u)};
        const u32x2 odd = {__builtin_amdgcn_perm(x1, x0, 0x07060302u),
                           __builtin_amdgcn_perm(x3, x2, 0x07060302u)};
        u32x2 *to = reinterpret_cast<u32x2 *>(&page.unit[quarter][g % 2][r]) + g / 2;
        to[2 * 16 * (2 * B)] = even;
        to[2 * 16 * (2 * B + 1)] = odd;
        store_values<E, D, B + 1, SAT>(page, x, quarter, r, g);
    }
}

// Queries of 32 rows as second operands: lane (n, h) holds, of row n, channels
// 64c + 16h .. +15 and 64c + 32 + 16h .. +15, in pieces.
template <typename E, int D>
struct Queries {
    static constexpr int kChunks = D / 64;
    i32x8 piece[E::kPieces][kChunks];
    uint32_t scale[kChunks];   // byte p: the scale of piece p of group 2c + h
};

template <typename E, int D>
__device__ __forceinline__ void load_queries(Queries<E, D> &q, const typename E::T *row, bool valid,
                                             int h) {
    u32x4 w[D / 64][2][2];
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            w[c][k][0] = w[c][k][1] = u32x4{0, 0, 0, 0};
            if (valid) {
                const u32x4 *at =
                    reinterpret_cast<const u32x4 *>(row + 64 * c + 32 * k + 16 * h);
                w[c][k][0] = at[0], w[c][k][1] = at[1];
            }
        }
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        float tops[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t x = w[c][k][i / 4][i % 4];
                bits = max(bits, max(x & 0x7FFFu, x >> 16 & 0x7FFFu));
            }
            const f32x2 both = both_halves(top_of<E>(bits));
            tops[k] = fmaxf(both[0], both[1]);
            const float up = group_scale<E>(tops[k]).up;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const auto pair = bits_as<typename E::T2>((uint32_t)w[c][k][i / 2][i % 2 * 2 + j / 2]);
                    y[j] = (float)pair[j % 2] * up;
                }
#pragma unroll
                for (int p = 0; p < E::kPieces; ++p) q.piece[p][c][4 * k + i] = (int)next_piece(y);
            }
        }
        q.scale[c] = group_scale<E>(h ? tops[1] : tops[0]).bytes;
    }
}

// A chunk's products of piece P, and those of the pieces after it.
template <typename E, int D, int T, int P>
__device__ __forceinline__ f32x16 multiply(const i32x8 &k, uint32_t scale, const Queries<E, D> &q,
                                           int c, f32x16 s) {
    if constexpr (P < E::kPieces) {
        s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q.piece[P][c], s, 4, 0, 2 * T,
                                                            (int)scale, P, (int)q.scale[c]);
        return multiply<E, D, T, P + 1>(k, scale, q, c, s);
    }
    return s;
}

// Scores of tokens 32T .. 32T + 31 of a page: s[i] of lane (n, h) is row n against
// token 32T + 8 (i / 4) + 4h + i % 4.
// The scales are shifted by the lane here, where the loads have to have come anyway: at the
// load it would wait for them a page early (216 -> 207 us, see the kernel).
template <typename E, int D, int T>
__device__ __forceinline__ f32x16 scores(const Keys<D> &r, const Queries<E, D> &q, int n) {
    f32x16 s = {};
#pragma unroll
    for (int c = 0; c < Keys<D>::kChunks; ++c) {
        const u32x4 k = r.k[T][c];
        s = multiply<E, D, T, 0>(i32x8{(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0},
                                 r.scale[c] >> (n / 16 * 8), q, c, s);
    }
    return s;
}

__device__ __forceinline__ float across_halves(float x, bool sum) {
    const f32x2 both = both_halves(x);
    return sum ? both[0] + both[1] : fmaxf(both[0], both[1]);
}

// Orders what stands since the last scheduling barrier: four LDS reads, then COUNT
// times VALU vector instructions, one matrix instruction and one more read.
template <int COUNT, int VALU>
__device__ __forceinline__ void interleave() {
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x002, VALU, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
}

// LDS operations of this wave done, then all waves here; loads from memory may
// stay on their way.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace

// Grid (tiles * kv_heads, splits), four waves of 32 rows.  Rows are the queries of
// one sequence times the heads that share the cache head.  Every wave multiplies
// all keys of a page, in 4 bits as they come from memory, by its own queries; the
// values are made into two-byte floats once a workgroup, a quarter by each wave, and
// read from LDS by all four.  Heads of 64 and 128 channels: of 256, a wave's state
// and queries leave no registers for a second wave (0.4 of the rate).
//
// Bound by issue: of a CU's busy cycles the matrix pipe is at work in 0.51 and the vector
// pipe in 0.57 (counters of the 6000-token case below), with two waves a SIMD to fill each
// other's gaps.  Measured, bfloat16, 32 heads on 8 of 128 channels, causal: 4 sequences of
// up to 2048 new tokens on up to 16384, 681 us, 1142 TFLOP/s of visible pairs (a large
// library product: 1217); of up to 1777 on up to 6000, 190 to 206 us by the card, up to
// 1068 TFLOP/s.  float16 has three pieces of a query to multiply instead of two: 776 us;
// heads of 64 the same softmax for half the products: 462 us, 842 TFLOP/s (float16 484).
template <typename E, int D>
__global__ __launch_bounds__(kThreads, 2) void attend128_kernel(AttendParams p) {
    __shared__ Page<D> pages[2];
    __shared__ int last;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % p.kv_heads, split = blockIdx.y;
    // the last tiles of a sequence see the most: they start first
    const int slot = (int)gridDim.x / p.kv_heads - 1 - (int)blockIdx.x / p.kv_heads;

    const auto first = [&](int s, int b) { return (int64_t)s * p.group / kRows + b; };
    const Sequence seq =
        find_sequence(p.q_start, p.lengths, p.seqs, p.tokens, p.width, slot, first);
    if (seq.index < 0) return;
    const int rows = seq.queries * p.group;
    const int row0 = (int)(slot - first(seq.start, seq.index)) * kRows;
    if (row0 >= rows) return;
    const int valid = min(rows - row0, kRows);
    const int row = row0 + kWaveRows * wave + n;
    const bool mine = row < rows;
    const int i = row / p.group, hq = head * p.group + row % p.group;
    const Span span = visible(seq, i, p.causal, p.window);
    // spans move up with the rows: the tile's, and this wave's, first and last
    const Span a = visible(seq, row0 / p.group, p.causal, p.window);
    const Span z = visible(seq, (row0 + valid - 1) / p.group, p.causal, p.window);
    const int row1 = min(row0 + kWaveRows * wave, rows - 1);
    const int row2 = min(row0 + kWaveRows * wave + kWaveRows, rows) - 1;
    const Span wa = visible(seq, row1 / p.group, p.causal, p.window);
    const Span wz = visible(seq, max(row1, row2) / p.group, p.causal, p.window);

    const int page0 = a.lo / kPage;
    const int count = z.hi > a.lo ? (z.hi + kPage - 1) / kPage - page0 : 0;
    const int splits = clampi((count + p.chunk - 1) / p.chunk, 1, (int)gridDim.y);
    if (split >= splits) return;
    const int end = split == splits - 1 ? count : (split + 1) * p.chunk;

    Queries<E, D> q;
    load_queries<E, D>(q,
                       (const typename E::T *)p.q + (int64_t)(seq.start + i) * p.q_token +
                           (int64_t)hq * p.q_head,
                       mine, h);

    // the state of a row: running maximum (log2), this lane's share of the sum, sums
    // of weighted values: o[m][i] is place 32m + 8 (i / 4) + 4h + i % 4
    float top = kNone, l = 0.0f;
    f32x16 o[D / 32];
#pragma unroll
    for (int m = 0; m < D / 32; ++m) o[m] = f32x16{};

    const int32_t *table = p.table + (int64_t)seq.index * p.width;
    const int64_t stride = (int64_t)p.kv_heads * Record<D>::kBytes;
    const uint8_t *cache = p.cache + (int64_t)head * Record<D>::kBytes;
    // 64 pages at a time, one a lane; the same in every wave
    int from = split * p.chunk, page = -1, phys = -1;
    uint64_t todo = 0;
    const auto fetch = [&]() {
        while (!todo && from < end) {
            page = page0 + from + lane;
            phys = from + lane < end ? table[page] : -1;
            from += 64;
            todo = __builtin_amdgcn_ballot_w64(phys >= 0 && phys < p.pages);
        }
    };
    const auto next = [&](int &number) {
        const int at = __builtin_ctzll(todo);
        todo &= todo - 1;
        number = __builtin_amdgcn_readlane(page, at);
        return cache + (int64_t)__builtin_amdgcn_readlane(phys, at) * stride;
    };
    const int r = lane & 15, g = lane >> 4;
    Keys<D> keys;
    Values<D> values;
    int number = 0, following = 0, now = 0;
    const auto load = [&](int &of) {
        const uint8_t *rec = next(of);
        keys.load(rec, n, h);
        values.load(rec, wave, r, g);
    };
    const auto settle = [&](int of) {
        const int t0 = of * kPage;
        if (t0 < z.lo || t0 + kPage > a.hi)
            values.scale = settled(values.scale, 16 * wave + 4 * g, a.lo - t0, z.hi - t0);
    };
    // whether the wave's quarter of a page has values past float16's range; it is then
    // stored once more, behind the ordinary place, the order of which a branch would break
    const auto past_range = [&]() {
        if constexpr (!E::kSaturates) return false;
        return __builtin_amdgcn_ballot_w64(past_float16(values.scale) != 0) != 0;
    };
    bool past = false;
    const auto saturate = [&](Page<D> &page) {
        if (__builtin_expect(past, 0)) store_values<E, D, 0, E::kSaturates>(page, values, wave, r, g);
    };
    // weights of 16 scores, two second operands of 16 tokens each; summed by themselves:
    // a long sequence's many small ones would be rounded one by one to the last place of
    // a large sum
    f32x16 s[2];
    u32x4 w[4];
    const auto weigh = [&](int t, float c) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; k += 2) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][k], c, -top));
            const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][k + 1], c, -top));
            sum += x;
            sum += y;
            w[2 * t + k / 8][k % 8 / 2] = pack_pair<E>(x, y);
        }
        l += sum;
    };
    const auto add = [&](int t) {
#pragma unroll
        for (int b = 2 * t; b < 2 * t + 2; ++b)
#pragma unroll
            for (int m = 0; m < D / 32; ++m)
                o[m] = E::mfma32(pages[now].unit[b][h][32 * m + n], w[b], o[m]);
    };

    // In the loop, s holds the scores of one page, LDS its values, and the registers
    // the keys and values of the next (of a page before, where there is none: what
    // is made of them is not used).  Matrix and vector instructions of independent
    // work are put next to each other: the second half's weights beside the first
    // half's products and the next page's scores, the next page's values beside the
    // rest.
    fetch();
    bool more = todo != 0;
    const bool any = more;
    if (any) {
        load(number);
        settle(number);
        store_values<E, D, 0>(pages[0], values, wave, r, g);
        past = past_range();
        saturate(pages[0]);
        s[0] = scores<E, D, 0>(keys, q, n);
        s[1] = scores<E, D, 1>(keys, q, n);
        fetch();
        more = todo != 0;
        if (more) load(following);
    }
    while (any) {
        lds_barrier();
        const int t0 = number * kPage;
        if (more) settle(following);
        if (t0 < wz.hi && t0 + kPage > wa.lo) {
            if (t0 < wz.lo || t0 + kPage > wa.hi) {
                const int lo = span.lo - t0 - 4 * h, hi = span.hi - t0 - 4 * h;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const int j = 32 * t + 8 * (k / 4) + k % 4;
                        s[t][k] = j >= lo && j < hi ? s[t][k] : -__builtin_inff();
                    }
            }
            float high = s[0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < 16; ++k) high = fmaxf(high, s[t][k]);
            high *= p.scale_log2;
            // (of large maxima, the difference is exact where a sum is not; each row goes by
            // its own maximum, so that no bit of it depends on the rows beside it)
            if (__builtin_amdgcn_ballot_w64(high - top > kLag + E::kLift)) {
                high = across_halves(high, false);
                const float all = high - top > kLag + E::kLift ? high - E::kLift : top;
                const float f = __builtin_amdgcn_exp2f(top - all);
                top = all;
                l *= f;
#pragma unroll
                for (int m = 0; m < D / 32; ++m) o[m] *= f;
            }
            // the fused product differs from the rounded one that the maximum is: where
            // that could show, round the scores' products too
            float c = p.scale_log2;
            const bool large = __builtin_fabsf(top) > kLarge;
            if (__builtin_amdgcn_ballot_w64(large)) {
                s[0] = large ? s[0] * c : s[0];
                s[1] = large ? s[1] * c : s[1];
                c = large ? 1.0f : c;
            }
            weigh(0, c);
            __builtin_amdgcn_sched_barrier(0);
            // The two waves of a SIMD are at different places of a page: the one at its
            // products goes first, or the other's softmax holds them up (207 -> 187 us).
            __builtin_amdgcn_s_setprio(1);
            add(0);
            s[0] = scores<E, D, 0>(keys, q, n);
            weigh(1, c);
            interleave<D / 16 + Keys<D>::kChunks * E::kPieces, 6>();
            __builtin_amdgcn_sched_barrier(0);
            add(1);
            past = past_range();
            s[1] = scores<E, D, 1>(keys, q, n);
            store_values<E, D, 0>(pages[now ^ 1], values, wave, r, g);
            interleave<D / 16 + Keys<D>::kChunks * E::kPieces, 4>();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
        } else {
            s[0] = scores<E, D, 0>(keys, q, n);
            s[1] = scores<E, D, 1>(keys, q, n);
            past = past_range();
            store_values<E, D, 0>(pages[now ^ 1], values, wave, r, g);
        }
        saturate(pages[now ^ 1]);
        if (!more) break;
        now ^= 1;
        number = following;
        fetch();
        more = todo != 0;
        if (more) load(following);
    }
    l = across_halves(l, true);

    // channel D/16 * r + c is at place 16c + r: register c / 2, element (c % 2 * 2 + r /
    // 8) * 4 + r % 4 of the half r / 4 % 2
    typedef Part<D, kRows> P;
    if (splits == 1) {
        if (!mine) return;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const int64_t at = (int64_t)(seq.start + i) * (p.kv_heads * p.group) + hq;
        typename E::T *out = (typename E::T *)p.out + at * D + D / 16 * 4 * h;
#pragma unroll
        for (int u = 0; u < 8; ++u) {   // r = 8 (u / 4) + 4h + u % 4
            uint32_t x[D / 32];
#pragma unroll
            for (int c = 0; c < D / 16; c += 2)
                x[c / 2] = pack_result<E>(o[c / 2][u / 4 * 4 + u % 4] * inv,
                                          o[c / 2][(2 + u / 4) * 4 + u % 4] * inv);
            typename E::T *to = out + D / 16 * (8 * (u / 4) + u % 4);
#pragma unroll
            for (int k = 0; k < D / 32; k += 2)
                *reinterpret_cast<u32x2 *>(to + 2 * k) = u32x2{x[k], x[k + 1]};
        }
        if (p.lse && h == 0)
            p.lse[at] = l == 0.0f ? -__builtin_inff()
                                  : (top + __builtin_log2f(l)) * 0.69314718055994531f;
        return;
    }

    // several splits: as in the kernel for 16 rows
    float *part = p.part + (int64_t)blockIdx.x * gridDim.y * P::kFloats;
    float *my = part + (int64_t)split * P::kFloats;
    const int at_row = kWaveRows * wave + n;
    if (mine) {
        if (h == 0) put(my + P::state(at_row), f32x2{top, l});
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int c = 0; c < D / 16; c += 4) {   // channels D/16 * r + c .. c + 3
                const int quad = (8 * (u / 4) + 4 * h + u % 4) * (D / 64) + c / 4;
                float *to = my + P::sums(kRows, at_row, quad);
                const int lo = u / 4 * 4 + u % 4, hi = (2 + u / 4) * 4 + u % 4;
                put(to, f32x2{o[c / 2][lo], o[c / 2][hi]});
                put(to + 2, f32x2{o[c / 2 + 1][lo], o[c / 2 + 1][hi]});
            }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) last = last_of(p.tickets + (int64_t)blockIdx.x * kTicketStride, splits);
    __syncthreads();
    if (!last) return;
    for (int x = threadIdx.x; x < kRows * (D / 4); x += kThreads) {
        const int rr = x % kRows, quad = x / kRows;
        if (rr >= valid) continue;
        float m, sum;
        const f32x4 v = join_splits<D, kRows>(part, splits, kRows, rr, quad, m, sum);
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int64_t at =
            (int64_t)(seq.start + (row0 + rr) / p.group) * (p.kv_heads * p.group) +
            head * p.group + (row0 + rr) % p.group;
        *reinterpret_cast<u32x2 *>((typename E::T *)p.out + at * D + 4 * quad) =
            u32x2{pack_result<E>(v[0] * inv, v[1] * inv), pack_result<E>(v[2] * inv, v[3] * inv)};
        if (p.lse && quad == 0)
            p.lse[at] = sum == 0.0f ? -__builtin_inff()
                                    : (m + __builtin_log2f(sum)) * 0.69314718055994531f;
    }
}

namespace {

template <typename E>
void launch_t(const AttendParams &p, int dim, dim3 grid, hipStream_t s) {
    if (dim == 64)
        hipLaunchKernelGGL((attend128_kernel<E, 64>), grid, dim3(kThreads), 0, s, p);
    else
        hipLaunchKernelGGL((attend128_kernel<E, 128>), grid, dim3(kThreads), 0, s, p);
}

}  // namespace

void launch_attend128(const AttendParams &p, int type, int dim, dim3 grid, hipStream_t s) {
    if (type == LCE_FLOAT16) launch_t<F16>(p, dim, grid, s);
    else launch_t<Bf16>(p, dim, grid, s);
}

}  // namespace kv4
}  // namespace lce
