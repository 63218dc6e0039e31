// Attention over the 8-bit cache, 128 query rows a tile: prompts.
#include "kv8_attend.hpp"

namespace lce {
namespace kv8 {
namespace {

constexpr int kWaves = kThreads / 64;
constexpr int kWaveRows = 32;
constexpr int kRows = kWaves * kWaveRows;
static_assert(kWaves == kBlocks, "a wave makes one block of the values into two-byte floats");

// One wave's block of a page's keys as they come from memory: lane (r, f) holds of token
// r channels 64c + 16f .. +15.
template <int D>
struct Keys {
    u32x4 k[D / 64];

    __device__ __forceinline__ void load(const uint8_t *rec, int block, int r, int f) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
            k[c] = *reinterpret_cast<const u32x4 *>(rec + Record<D>::kKey +
                                                    (kBlock * block + r) * D + 64 * c + 16 * f);
    }
};

// One wave's block of a page's values: lane (r, g) holds tokens 4g .. 4g + 3 of channels
// 64c + 4r .. +3, a word for each channel.
template <int D>
struct Values {
    u32x4 v[D / 64];

    __device__ __forceinline__ void load(const uint8_t *rec, int block, int r, int g) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
            v[c] = *reinterpret_cast<const u32x4 *>(rec + Record<D>::kValue +
                                                    (4 * block + g) * 4 * D + (64 * c + 4 * r) * 4);
    }
};

// A page in LDS, two bytes a value, in the order in which the products read it, so that a
// wave's reads and writes are runs of memory and places differ by constants.  Values: for 16
// tokens at a time and each half of the wave, 16 bytes for each channel, of tokens 4h ..
// 4h + 3 and 8 + 4h .. 8 + 4h + 3 (those whose scores the half has); channel 64c + 4r + x at
// place 64c + 16x + r.  Keys: for every eight channels 16 bytes a token.
template <int D>
struct Page {
    u32x4 unit[kBlocks][2][D];
    u32x4 piece[D / 8][kPage];

    // the keys of channels 64c + 16f .. +15 of a block's token r
    template <typename E>
    __device__ __forceinline__ void store_keys(const Keys<D> &k, float scale, int block, int r,
                                               int f, int c) {
        piece[8 * c + 2 * f][kBlock * block + r] =
            decode_eight<E>(k.k[c][0], k.k[c][1], scale, scale);
        piece[8 * c + 2 * f + 1][kBlock * block + r] =
            decode_eight<E>(k.k[c][2], k.k[c][3], scale, scale);
    }
    // the values of channels 64c + 4r + x of its tokens 4g .. 4g + 3
    template <typename E>
    __device__ __forceinline__ void store_values(const Values<D> &v, float scale, int block, int r,
                                                 int g, int c, int x) {
        u32x2 *to = reinterpret_cast<u32x2 *>(&unit[block][g % 2][64 * c + 16 * x + r]);
        to[g / 2] = u32x2{decode_codes<E, false>(v.v[c][x], scale),
                          decode_codes<E, true>(v.v[c][x], scale)};
    }
};

// Queries of 32 rows as second operands: lane (n, h), n = lane % 32, h = lane / 32, holds
// of row n channels 16j + 8h .. +7.
template <int D>
struct Queries {
    u32x4 q[D / 16];

    __device__ __forceinline__ void load(const uint16_t *row, bool valid, int h) {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            q[j] = u32x4{0, 0, 0, 0};
            if (valid) q[j] = *reinterpret_cast<const u32x4 *>(row + 16 * j + 8 * h);
        }
    }
    template <typename E>
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) q[j][x] = without_infinities<E>(q[j][x]);
    }
};

__device__ __forceinline__ float across_halves(float x, bool sum) {
    const f32x2 both = both_halves(x);
    return sum ? both[0] + both[1] : fmaxf(both[0], both[1]);
}

// Weights are made here, not where they are used, which is in another block.
__device__ __forceinline__ void pin(u32x4 &a, u32x4 &b, float &c) {
    asm volatile("" : "+v"(a), "+v"(b), "+v"(c));
}

// LDS operations of this wave done, then all waves here; loads from memory may
// stay on their way.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace

// Grid (tiles * kv_heads, splits), four waves of 32 rows.  Rows are the queries of one
// sequence times the heads that share the cache head.  A page's keys and values are made
// into two-byte floats once a workgroup, a block by each wave, and read from LDS by all four.
// (From memory in the order of the products, keys are 32 pieces of lines a load, and with
// conversions in every wave, 8-bit keys through LDS gained nothing: 590 us of the first
// case below each, 550 now.  8-bit products of keys and queries in 8-bit pieces would need
// no conversion, but sum with fewer bits than float32: scores of 350 are off by 6e-3,
// against 3e-5.)
//
// Bound by issue: of a CU's busy cycles the matrix pipe is at work in 0.49 and the vector
// pipe in 0.59 (counters of the first case).  With two waves a SIMD the sum hardly passes 1:
// a matrix instruction holds up about six vector ones, measured alone (32x32x16 products
// with 8, 12 and 16 independent fused multiply-adds each: 21, 28 and 33 ns, 15 without).
// Measured, bfloat16, 32 heads on 8 of 128 channels: 4096 tokens seeing 8192, 550 to 558 us,
// 985 to 999 TFLOP/s; 4 sequences of up to 2048 new tokens on up to 16384, causal, 887 to 998
// TFLOP/s of visible pairs, by how alike their lengths are (a large library product: 1170 to
// 1390); of up to 1700 on up to 6500, of which one has 85 % of the work, 196 to 204 us, 875
// to 910 TFLOP/s, by the card.
template <typename E, int D, Change CHANGE>
__global__ __launch_bounds__(kThreads, 2) void attend128_kernel(AttendParams p) {
    __shared__ Page<D> pages[2];
    __shared__ int last;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % p.kv_heads, split = blockIdx.y;
    const int slot = (int)blockIdx.x / p.kv_heads;

    const auto first = [&](int s, int b) { return (int64_t)s * p.group / kRows + b; };
    const Sequence seq =
        find_sequence(p.q_start, p.lengths, p.seqs, p.tokens, p.width, slot, first);
    if (seq.index < 0) return;
    const int rows = seq.queries * p.group;
    // the last tiles of a sequence see the most: they start first
    const int tile = (rows + kRows - 1) / kRows - 1 - (int)(slot - first(seq.start, seq.index));
    if (tile < 0) return;
    const int row0 = tile * kRows;
    const int valid = min(rows - row0, kRows);
    const int row = row0 + kWaveRows * wave + n;
    const bool mine = row < rows;
    const int i = row / p.group, hq = head * p.group + row % p.group;
    const int prefix = p.prefix ? p.prefix[seq.index] : 0;
    const auto sees = [&](int query) { return visible(seq, query, p.causal, p.window, prefix); };
    const Span span = sees(i);
    // spans move up with the rows: the tile's, and this wave's, first and last
    const Span a = sees(row0 / p.group), z = sees((row0 + valid - 1) / p.group);
    const int row1 = min(row0 + kWaveRows * wave, rows - 1);
    const int row2 = min(row0 + kWaveRows * wave + kWaveRows, rows) - 1;
    const Span wa = sees(row1 / p.group), wz = sees(max(row1, row2) / p.group);

    const int page0 = a.lo / kPage;
    const int count = z.hi > a.lo ? (z.hi + kPage - 1) / kPage - page0 : 0;
    const int splits = clampi((count + p.chunk - 1) / p.chunk, 1, (int)gridDim.y);
    if (split >= splits) return;
    const int end = split == splits - 1 ? count : (split + 1) * p.chunk;

    Queries<D> q;
    q.load((const uint16_t *)p.q + (int64_t)(seq.start + i) * p.q_token + (int64_t)hq * p.q_head,
           mine, h);
    const Cap cap = {p.cap_log2, p.cap_inverse};
    Slope slope;
    if constexpr (has_slopes(CHANGE))
        slope.set(p.slopes && mine ? p.slopes[hq] : 0.0f, seq.length - seq.queries + i);

    // the state of a row: running maximum (log2), this lane's share of the sum, sums of
    // weighted values and their scale: o[m][i] is place 32m + 8 (i / 4) + 4h + i % 4
    float top = kNone, l = 0.0f;
    int biggest = kLeastScale;
    f32x16 o[D / 32];
#pragma unroll
    for (int m = 0; m < D / 32; ++m) o[m] = f32x16{};

    const int32_t *table = p.table + (int64_t)seq.index * p.width;
    const int64_t stride = (int64_t)p.kv_heads * Record<D>::kBytes;
    const uint8_t *cache = p.cache + (int64_t)head * Record<D>::kBytes;
    // 64 pages at a time, one a lane; the same in every wave
    int from = split * p.chunk, page = -1, phys = -1;
    uint64_t todo = 0;
    const auto look = [&]() {
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
    // the lane's token of a block of keys and its channels; its channels of a block of values
    // and their tokens (neighbouring lanes write the two halves of 16 bytes)
    const int kr = lane & 15, kq = lane >> 4, r = lane >> 1 & 15, g = (lane & 1) * 2 + (lane >> 5);
    Keys<D> keys;
    Values<D> values;
    // of the page whose keys the registers hold, and of the one before it, whose values they do
    u32x2 scales = {0, 0};
    uint32_t value_scales = 0;
    // What becomes of a page: the factor of its scores, of this wave's block of its keys, the
    // scale of its values and the factor of this wave's block.  Every wave comes to the same
    // for the page.
    float c = 1.0f, kf = 1.0f, vf = 1.0f;
    int held = kLeastScale;                    // scale of the values that were stored last
    const auto edge = [&](int of) {            // whether some row does not see all of a page
        return of * kPage < z.lo || of * kPage + kPage > a.hi;
    };
    const auto settled = [&](uint32_t scales, int of) {
        const uint32_t x = in_scalar(scales);
        return edge(of) ? settled_scales(x, a.lo - of * kPage, z.hi - of * kPage) : x;
    };
    const auto settle_keys = [&](int of) {
        const uint32_t ks = settled(scales[0], of);
        const int km = largest_of(ks);
        c = score_factor<E>(p.scale_log2, km);
        kf = relative(byte_of(ks, wave), km, kUp<E>);
    };
    const auto settle_values = [&](int of) {
        const uint32_t vs = settled(value_scales, of);
        held = max(held, largest_of(vs));
        vf = relative(byte_of(vs, wave), held, kUp<E>);
    };
    const auto clear = [&](int of) {
        const int t0 = of * kPage;
        if (edge(of)) {
            const uint32_t mask = seen_bytes(16 * wave + 4 * g, a.lo - t0, z.hi - t0);
#pragma unroll
            for (int x = 0; x < D / 64; ++x) values.v[x] &= mask;
        }
    };
    int now = 0;                               // which LDS buffer holds the page at hand
    f32x16 s[2];
    float factor[2];                           // what s is multiplied by, and then, by the cap,
    float offset = 0.0f;                       // what is added
    u32x4 w[4];                                // weights: second operands of 16 tokens each
    const auto add = [&](int t) {
#pragma unroll
        for (int b = 2 * t; b < 2 * t + 2; ++b)
#pragma unroll
            for (int m = 0; m < D / 32; ++m)
                o[m] = E::mfma32(pages[now].unit[b][h][32 * m + n], w[b], o[m]);
    };
    // Scores of half t of a page into the row's maximum, while the weights of the half
    // before, against the maximum so far, wait to be added.
    const auto judge = [&](int t, int of, float by, bool there) {
        const int t0 = of * kPage + 32 * t;
        const auto all = [&](auto f) {
#pragma unroll
            for (int k = 0; k < 16; ++k) s[t][k] = f(s[t][k], 8 * (k / 4) + k % 4);
        };
        if (CHANGE == Change::kCapped || (CHANGE == Change::kAny && cap.cap > 0.0f))
            cap.limit<CHANGE>(by, offset,
                              [&](auto f) { all([&](float x, int) { return f(x); }); });
        if (CHANGE == Change::kSloped || (CHANGE == Change::kAny && p.slopes)) {
            const float far = slope.from(t0 + 4 * h);
            all([&](float x, int j) { return slope(x * by, far - (float)j); });
            by = 1.0f;
        }
        if (!there || t0 < wz.lo || t0 + 32 > wa.hi) {
            const int lo = span.lo - t0 - 4 * h, hi = there ? span.hi - t0 - 4 * h : lo;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int j = 8 * (k / 4) + k % 4;
                s[t][k] = j >= lo && j < hi ? s[t][k] : -__builtin_inff();
            }
        }
        float high = s[t][0];
#pragma unroll
        for (int k = 1; k < 16; ++k) high = fmaxf(high, s[t][k]);
        high = __builtin_fmaf(high, by, offset);
        // (of large maxima, the difference is exact where a sum is not; each row goes by
        // its own maximum, so that no bit of it depends on what the rows beside it hold)
        if (__builtin_amdgcn_ballot_w64(high - top > kLag + E::kLift)) {
            add(t ^ 1);
            w[2 * (t ^ 1)] = w[2 * (t ^ 1) + 1] = u32x4{0, 0, 0, 0};
            high = across_halves(high, false);
            const float all = high - top > kLag + E::kLift ? high - E::kLift : top;
            const float f = __builtin_amdgcn_exp2f(top - all);
            top = all;
            l *= f;
#pragma unroll
            for (int m = 0; m < D / 32; ++m) o[m] *= f;
        }
        // the fused product differs from the rounded one that the maximum is: where that
        // could show, round the scores' products too
        const bool large = CHANGE != Change::kCapped && __builtin_fabsf(top) > kLarge;
        if (CHANGE != Change::kCapped && __builtin_amdgcn_ballot_w64(large)) {
            s[t] = large ? s[t] * by : s[t];
            by = large ? 1.0f : by;
        }
        factor[t] = by;
    };
    // The weights of scores k and k + 1 of half t.
    const auto weigh = [&](int t, int k, float &sum) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][k], factor[t], offset - top));
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][k + 1], factor[t], offset - top));
        sum += x;
        sum += y;
        w[2 * t + k / 8][k % 8 / 2] = pack_pair<E>(x, y);
    };
    // Half t of the page at hand is added and half t of the next one multiplied by the
    // queries, while the weights of the other half (of the page at hand, or of the next) are
    // made, which are summed by themselves: a long sequence's many small ones would be
    // rounded one by one to the last place of a large sum.  In each step one product of
    // either kind, the codes of the next, and as many weights; in the second half's steps a
    // share of the next page's values, too.
    constexpr int kSteps = D / 16, kWidth = D / 32;
    // first operand j of half t of a page's keys
    const auto key = [&](const Page<D> &from, int t, int j) {
        return from.piece[2 * j + h][32 * t + n];
    };
    const auto value = [&](int t, int j) {
        return pages[now].unit[2 * t + j / kWidth][h][32 * (j % kWidth) + n];
    };
    // the operands of a phase's first steps are on their way while its scores are judged
    u32x4 k[3], v[3];
    const auto begin = [&](int t) {
#pragma unroll
        for (int j = 0; j < 2; ++j) k[j] = key(pages[now ^ 1], t, j), v[j] = value(t, j);
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto phase = [&](int t) {
        Page<D> &ours = pages[now], &other = pages[now ^ 1];
        float sum = 0.0f;
        f32x16 next = {};
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            if (j + 2 < kSteps) {
                k[(j + 2) % 3] = key(other, t, j + 2);
                v[(j + 2) % 3] = value(t, j + 2);
            }
            next = E::mfma32(k[j % 3], q.q[j], next);
            if (t == 0 && j % 4 == 1)
                ours.template store_keys<E>(keys, kf, wave, kr, kq, j / 4);
            if (t == 1) other.template store_values<E>(values, vf, wave, r, g, j / 4, j % 4);
            o[j % kWidth] = E::mfma32(v[j % 3], w[2 * t + j / kWidth], o[j % kWidth]);
#pragma unroll
            for (int x = 16 / kSteps * j; x < 16 / kSteps * (j + 1); x += 2) weigh(t ^ 1, x, sum);
            __builtin_amdgcn_sched_barrier(0);
        }
        l += sum;
        s[t] = next;
        pin(w[2 * (t ^ 1)], w[2 * (t ^ 1) + 1], l);
    };

    // In the loop, LDS holds the values of one page and the keys of the next, w the weights
    // of the page's first half and s the scores of its second; the registers hold the values
    // of the next page and the keys of the one after it.  What there is no page for is made
    // of what was there before, and not used.
    int number[4];                             // the page at hand and the next ones, or -1
    const uint8_t *rec[4];
    const auto pull = [&](int at) {
        look();
        number[at] = -1;
        if (todo) rec[at] = next(number[at]);
    };
    const auto load_keys = [&](const uint8_t *from) {
        value_scales = scales[1];
        scales = *reinterpret_cast<const u32x2 *>(from + Record<D>::kScale);
        keys.load(from, wave, kr, kq);
    };
    const auto store_keys = [&](Page<D> &page) {
#pragma unroll
        for (int x = 0; x < D / 64; ++x) page.template store_keys<E>(keys, kf, wave, kr, kq, x);
    };
    pull(0);
    const bool any = number[0] >= 0;
    float factor0 = 1.0f, factor1 = 1.0f;      // c of the page at hand and of the next
    if (any) {
        pull(1);
        pull(2);
        load_keys(rec[0]);
        values.load(rec[0], wave, r, g);
        settle_keys(number[0]);
        factor0 = c;
        store_keys(pages[0]);
        if (number[1] >= 0) {
            load_keys(rec[1]);
            settle_keys(number[1]);
            factor1 = c;
        } else {
            value_scales = scales[1];
        }
        settle_values(number[0]);
        clear(number[0]);
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
            pages[0].template store_values<E>(values, vf, wave, r, g, j / 4, j % 4);
        store_keys(pages[1]);
        if (number[1] >= 0) values.load(rec[1], wave, r, g);
        if (number[2] >= 0) load_keys(rec[2]);
        else value_scales = scales[1];
        q.template settle<E>();
        lds_barrier();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x16{};
#pragma unroll
            for (int j = 0; j < kSteps; ++j) s[t] = E::mfma32(key(pages[0], t, j), q.q[j], s[t]);
        }
        biggest = held;
        w[2] = w[3] = u32x4{0, 0, 0, 0};
        judge(0, number[0], factor0, true);
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; k += 2) weigh(0, k, sum);
        l += sum;
        lds_barrier();                         // all waves have these keys
    }
    while (any) {
        const int before = held;
        const bool more = number[1] >= 0;
        begin(0);
        if (number[2] >= 0) settle_keys(number[2]);
        if (more) {
            settle_values(number[1]);
            clear(number[1]);
        }
        judge(1, number[0], factor0, true);
        __builtin_amdgcn_sched_barrier(0);
        // The two waves of a SIMD are at different places of a page: the one at its
        // products goes first.
        __builtin_amdgcn_s_setprio(1);
        phase(0);
        __builtin_amdgcn_s_setprio(0);
        begin(1);
        pull(3);
        if (number[3] >= 0) load_keys(rec[3]);
        else value_scales = scales[1];
        judge(0, number[1], more ? factor1 : 1.0f, more);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        phase(1);
        __builtin_amdgcn_s_setprio(0);
        if (!more) break;
        if (number[2] >= 0) values.load(rec[2], wave, r, g);
        if (held > before) {
            const float f = relative(before, held, 0);
            biggest = held;
#pragma unroll
            for (int m = 0; m < D / 32; ++m) o[m] *= f;
        }
        factor0 = factor1;
        factor1 = c;
        now ^= 1;
#pragma unroll
        for (int x = 0; x < 3; ++x) number[x] = number[x + 1], rec[x] = rec[x + 1];
        lds_barrier();
    }
    l = across_halves(l, true);

    // channels 64c + 4r + x, x = 0 .. 3, r = 8 (u / 4) + 4h + u % 4, are element u and u + 8
    // of registers 2c and 2c + 1
    const auto four = [&](int c, int u) {
        return f32x4{o[2 * c][u], o[2 * c][u + 8], o[2 * c + 1][u], o[2 * c + 1][u + 8]};
    };
    const int64_t at = (int64_t)(seq.start + i) * (p.kv_heads * p.group) + hq;
    if (splits == 1) {
        if (!mine) return;
        typename E::T *out = (typename E::T *)p.out + at * D;
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int u = 0; u < 8; u += 2) {
                const int rr = 8 * (u / 4) + 4 * h + u % 4;
                const u32x2 x = result<E>(four(c, u), l, biggest);
                const u32x2 y = result<E>(four(c, u + 1), l, biggest);
                *reinterpret_cast<u32x4 *>(out + 64 * c + 4 * rr) = u32x4{x[0], x[1], y[0], y[1]};
            }
        if (p.lse && h == 0) p.lse[at] = log_sum(top, l);
        return;
    }

    // several splits: as in the kernel for 16 rows
    typedef Part<D, kRows> P;
    float *part = p.part + (int64_t)blockIdx.x * gridDim.y * P::kFloats;
    float *my = part + (int64_t)split * P::kFloats;
    const int at_row = kWaveRows * wave + n;
    if (mine) {
        if (h == 0) {
            put(my + P::state(at_row), f32x2{top, l});
            put(my + P::state(at_row) + 2, f32x2{(float)biggest, l});
        }
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int quad = 16 * c + 8 * (u / 4) + 4 * h + u % 4;
                float *to = my + P::sums(kRows, at_row, quad);
                const f32x4 x = four(c, u);
                put(to, f32x2{x[0], x[1]});
                put(to + 2, f32x2{x[2], x[3]});
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
        const Joined j = join_parts<D, kRows>(part, splits, kRows, rr, quad);
        const int64_t to =
            (int64_t)(seq.start + (row0 + rr) / p.group) * (p.kv_heads * p.group) +
            head * p.group + (row0 + rr) % p.group;
        *reinterpret_cast<u32x2 *>((typename E::T *)p.out + to * D + 4 * quad) =
            result<E>(j.o, j.divisor, j.scale);
        if (p.lse && quad == 0) p.lse[to] = log_sum(j.top, j.l);
    }
}

namespace {

template <typename E, int D>
void launch_d(const AttendParams &p, dim3 grid, hipStream_t s) {
    by_change(p, [&](auto kind) {
        hipLaunchKernelGGL((attend128_kernel<E, D, decltype(kind)::value>), grid, dim3(kThreads), 0,
                           s, p);
    });
}

template <typename E>
void launch_t(const AttendParams &p, int dim, dim3 grid, hipStream_t s) {
    if (dim == 64) launch_d<E, 64>(p, grid, s);
    else launch_d<E, 128>(p, grid, s);
}

}  // namespace

void launch_attend128(const AttendParams &p, int type, int dim, dim3 grid, hipStream_t s) {
    if (type == LCE_FLOAT16) launch_t<F16>(p, dim, grid, s);
    else launch_t<Bf16>(p, dim, grid, s);
}

}  // namespace kv8
}  // namespace lce
