// Attention over the 8-bit cache, 16 or 32 query rows a tile: single tokens, a few tokens,
// short prompts.
#include "kv8_attend.hpp"

namespace lce {
namespace kv8 {
namespace {

constexpr int kWaves = kThreads / 64;

// A load from the cache; ONCE: past the caches, of what nobody else will read soon.
template <bool ONCE, typename V>
__device__ __forceinline__ V fetch(const uint8_t *p) {
    if constexpr (ONCE)
        return __builtin_nontemporal_load(reinterpret_cast<const V *>(p));
    else
        return *reinterpret_cast<const V *>(p);
}

// What a wave takes at a time: T tiles of 16 tokens, a page or half of one.
template <int D, int T>
struct Step {
    static constexpr int kTiles = T;
    static constexpr int kPerPage = 4 / kTiles;
    static constexpr int kTokens = 16 * kTiles;
    static constexpr int kChunks = D / 64;
};

// Half a page where the codes of a whole one would leave too few registers for what else
// there is: wide heads (of 128: 67 us against 87 of 48 sequences of up to 8192 tokens, when
// keys did not come through LDS yet), and 32 rows of 64 with a cap and a bias (62 against 63
// us of the prompts below, if they had a bias; with their cap alone 49.5 against 46.6).
template <int D, int C, Change CHANGE>
constexpr int kTilesOf = D <= 64 && !(C == 2 && CHANGE == Change::kAny) ? 4 : 2;

// Key codes of a step as they come from memory, whole lines of it: 16 bytes a lane at a
// time, pieces lane, lane + 64 .. of the step's.  The wave's own part of LDS turns them into
// first operands: lane (n, g), n = lane % 16, g = lane / 16, wants piece 4c + g, 16 channels
// for two products, of tokens 16t + n (loads in that order are sixteen pieces of lines each,
// 67 against 59 us).  A token's pieces change places with its number, or they would meet in
// a bank.
template <int D, int T>
struct Keys {
    static constexpr int kPieces = D / 16, kLoads = T * D / 64;
    u32x4 k[kLoads];

    template <bool ONCE>
    __device__ __forceinline__ void load(const uint8_t *rec, int half, int lane) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            k[i] = fetch<ONCE, u32x4>(rec + Record<D>::kKey + half * Step<D, T>::kTokens * D +
                                      1024 * i + 16 * lane);
    }
    static __device__ __forceinline__ int place(int token, int piece) {
        constexpr int kApart = kPieces < 8 ? 4 : 1;
        return token * kPieces + (piece ^ (token / kApart % kPieces));
    }
    __device__ __forceinline__ void store(u32x4 *to, int lane) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = 64 * i + lane;
            to[place(at / kPieces, at % kPieces)] = k[i];
        }
    }
};

// Value codes: lane (n, g) holds of channels 64c + 4n .. +3 tokens 16t + 4g .. +3, a word
// for each channel.
template <int D, int T>
struct Values {
    u32x4 v[Step<D, T>::kTiles][Step<D, T>::kChunks];

    template <bool ONCE>
    __device__ __forceinline__ void load(const uint8_t *rec, int half, int n, int g) {
#pragma unroll
        for (int t = 0; t < Step<D, T>::kTiles; ++t)
#pragma unroll
            for (int c = 0; c < Step<D, T>::kChunks; ++c)
                v[t][c] = fetch<ONCE, u32x4>(
                    rec + Record<D>::kValue +
                    ((half * Step<D, T>::kTiles + t) * 4 + g) * 4 * D + (64 * c + 4 * n) * 4);
    }
    // what no row sees
    __device__ __forceinline__ void clear(int first, int lo, int hi) {
#pragma unroll
        for (int t = 0; t < Step<D, T>::kTiles; ++t) {
            const uint32_t mask = seen_bytes(first + 16 * t, lo, hi);
#pragma unroll
            for (int c = 0; c < Step<D, T>::kChunks; ++c) v[t][c] &= mask;
        }
    }
};

// Queries of 16 rows as second operands: lane (n, g) holds of row n the channels that it
// holds of the keys.
template <int D>
struct Queries {
    u32x4 q[D / 64][2];

    __device__ __forceinline__ void load(const void *row, bool valid, int g) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            q[c][0] = q[c][1] = u32x4{0, 0, 0, 0};
            if (valid) {
                const u32x4 *at = reinterpret_cast<const u32x4 *>(
                    static_cast<const uint16_t *>(row) + 64 * c + 16 * g);
                q[c][0] = at[0], q[c][1] = at[1];
            }
        }
    }
    template <typename E>
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int x = 0; x < 8; ++x)
                q[c][x / 4][x % 4] = without_infinities<E>(q[c][x / 4][x % 4]);
    }
};

// A row's state: running maximum of scores (log2), this lane's share of the sum and of what
// results are divided by, and the sums of weighted values: o[4c + x][i] of lane (n, g) is row n,
// channel 64c + 16g + 4i + x.
template <int D>
struct RowState {
    float m, l, divisor;
    f32x4 o[D / 16];
};

// The waves' states, where they are joined; before that, each wave's part holds its keys.
template <int D, int C>
struct Shared {
    f32x4 o[kWaves][D / 4][16 * C];
    f32x4 ml[kWaves][16 * C];                  // m, l, divisor
    int scale[kWaves];
    int last;
    static_assert(sizeof(o[0]) >= (D <= 64 ? 64 : 32) * D, "a step's keys");
};

// What a weight's rounding does to results shows most in rows that go by few tokens, and in
// calls of few rows (FEW: up to 64 of a sequence and cache head).  In tiles of up to 8 rows
// of such calls, the products' other eight columns, lanes n >= 8, take what is left of each
// weight once its leading bits, kCut, are cut off: results are as with float32 weights (errors
// against 64 bits 1.0 times those of rounding the result, with rounded weights 1.2 and up to
// 1.9; 0 to 2 % of a decoding step's time).  In their taller tiles they are divided by the sum
// of the rounded weights, so that a row that goes by one token has that token's values.  In
// the many rows of a prompt they are divided by the sum itself: the other would take 4 % of
// them in tiles of 16 rows, 3 of 32, 7 of 128.

// The bits of a float32 that are an E::T's.
template <typename E>
constexpr uint32_t kCut = __is_same(E, F16) ? 0xFFFFE000u : 0xFFFF0000u;

__device__ __forceinline__ float cut(float x, uint32_t mask) {
    return bits_as<float>(bits_as<uint32_t>(x) & mask);
}

// A pair of E::T, what they cannot hold cut off.
template <typename E>
__device__ __forceinline__ uint32_t cut_pair(float x, float y) {
    if constexpr (__is_same(E, F16))
        return bits_as<uint32_t>(__builtin_amdgcn_cvt_pkrtz(x, y));
    else
        return __builtin_amdgcn_perm(bits_as<uint32_t>(y), bits_as<uint32_t>(x), 0x07060302u);
}

// How far under the largest score (log2) weights are taken.  What is cut off of float16's
// smallest numbers is a whole last place, and not half of one: where weights are cut, the
// largest is 2^3 as large, for a maximum that moves a little more often.
template <typename E, bool FEW>
constexpr float kUnder = E::kLift + (FEW && E::kLift > 0.0f ? 3.0f : 0.0f);

// A step's scores into the rows' maximum and sum; its weights, ready to be multiplied.
// Scores times c, plus `offset`, are in log2 units.
template <typename E, int D, Change CHANGE, bool FEW, int kTiles>
__device__ __forceinline__ void weigh(RowState<D> &st, f32x4 (&s)[kTiles], u32x4 (&p)[kTiles / 2],
                                      float c, float offset, bool paired, uint32_t taken) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
    top = __builtin_fmaf(top, c, offset);
    // (Of large maxima, the difference is exact where a sum is not.  Each row goes by
    // its own maximum, so that no bit of it depends on what the rows beside it hold; how
    // many they are does count, by `paired`.)
    if (__builtin_amdgcn_ballot_w64(top - st.m > kLag + E::kLift)) {
        const float high = across_rows(top, [](float a, float b) { return fmaxf(a, b); });
        const float all = high - st.m > kLag + E::kLift ? high - kUnder<E, FEW> : st.m;
        const float f = __builtin_amdgcn_exp2f(st.m - all);
        st.m = all;
        st.l *= f;
        st.divisor *= f;
#pragma unroll
        for (int m = 0; m < D / 16; ++m) st.o[m] *= f;
    }
    // The fused product below differs from the rounded one that the maximum is: where
    // that could show (scores past kLarge), round the scores' products too.
    const bool large = CHANGE != Change::kCapped && __builtin_fabsf(st.m) > kLarge;
    if (CHANGE != Change::kCapped && __builtin_amdgcn_ballot_w64(large)) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) s[t] = large ? s[t] * c : s[t];
        c = large ? 1.0f : c;
    }
    // summed by themselves: a long sequence's many small ones would be rounded one by one
    // to the last place of a large sum
    float sum = 0.0f, rounded = 0.0f;
    const float minus = offset - st.m;
    float w[kTiles][4];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], c, minus));
            sum += w[t][i];
        }
    const auto pairs = [&](auto f) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                p[t / 2][t % 2 * 2 + i] = f(w[t][2 * i], w[t][2 * i + 1]);
    };
    if (FEW && paired) {
        pairs([&](float x, float y) { return cut_pair<E>(x - cut(x, taken), y - cut(y, taken)); });
    } else {
        pairs([](float x, float y) { return pack_pair<E>(x, y); });
        if constexpr (FEW) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    rounded = add_rounded(E(), p[t / 2][t % 2 * 2 + i], rounded);
        }
    }
    st.l += sum;
    st.divisor += FEW && !paired ? rounded : sum;
}

}  // namespace

// Grid (tiles * kv_heads, splits), four waves.  A tile is C times 16 rows of one head
// of the cache: rows are the queries of one sequence times the heads that share the cache
// head, in that order.  The waves take the pages of their workgroup's split in turn, each
// with all rows, and join their states at the end; the last split of a tile to finish
// joins all of them, in the order of the splits, so that results do not depend on timing.
//
// Keys are the first operand and queries the second, so that a lane's scores belong to one
// row and the weights leave the softmax as the second operand of the product with the
// values; no weight and no score crosses lanes.  Codes become two-byte floats in the
// conversion instruction, which multiplies them by their block's power of two as well: of
// the keys against the step's largest, which the scores are multiplied by in float32, of
// the values against the largest that the wave has seen.
//
// Bound by memory where a call reads much: 48 sequences of up to 8192 tokens, 32 heads of
// 128 on 8, bfloat16 (265 MB) 60 us, 4.4 TB/s with the launch (a large copy 4.8 to 5.4, by
// the card); 24 of up to 4001, 32 heads of 64 on 32 with a bias (170 MB) 36 us; 16 with 4
// drafted tokens and a window of 4096, 16 heads of 256 on 8, float16, capped (191 MB) 44 us.
// By latencies in a row (launch, lengths, table, a page, the states out, the ticket, the
// states in) where it does not: one of 30011, 32 heads of 128 on 8 (61 MB) 18 us.  A page
// more a wave is 0.8, 1.6 and 2.3 us in heads of 64, 128 and 256.  Prompts by instruction
// issue: three of up to 2500 tokens behind prefixes, 16 heads of 64 on 2, float16, capped,
// 42 to 47 us in tiles of 32 rows.
template <typename E, int D, int C, Change CHANGE, bool FEW, bool ONCE>
__global__ __launch_bounds__(kThreads, D == 64 || (D == 128 && C == 1) ? 3 : 2) void attend16_kernel(
    AttendParams p) {
    constexpr int kRows = 16 * C;
    typedef Step<D, kTilesOf<D, C, CHANGE>> S;
    __shared__ Shared<D, C> sh;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the eight XCDs in turn, and where the grid is a multiple of eight
    // wide all splits of a tile would go to one: tiles are moved on by one a split.
    const int split = blockIdx.y;
    int unit = blockIdx.x;
    if (p.turn) {
        unit += split % 8;
        if (unit >= p.turn) unit -= p.turn;
    }
    const int head = unit % p.kv_heads, slot = unit / p.kv_heads;

    // a sequence's tiles begin at floor(rows before it / kRows) + its index: at most one
    // more than it needs, and none shared
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
    const int prefix = p.prefix ? p.prefix[seq.index] : 0;
    const bool paired = FEW && valid <= 8;
    const uint32_t taken = paired && n >= 8 ? kCut<E> : 0u;
    const int nr = paired ? n & 7 : n;
    // this lane's row of each sixteen
    int i[C], hq[C];
    bool mine[C];
    Span span[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int row = row0 + 16 * c + nr;
        i[c] = row / p.group, hq[c] = head * p.group + row % p.group;
        mine[c] = 16 * c + nr < valid;
        span[c] = visible(seq, i[c], p.causal, p.window, prefix);
    }
    // spans move up with the rows: the tile's first and last row bound them
    const Span a = visible(seq, row0 / p.group, p.causal, p.window, prefix);
    const Span z = visible(seq, (row0 + valid - 1) / p.group, p.causal, p.window, prefix);

    // this workgroup's share of the pages
    const int page0 = a.lo / kPage;
    const int count = z.hi > a.lo ? (z.hi + kPage - 1) / kPage - page0 : 0;
    const int splits = clampi((count + p.chunk - 1) / p.chunk, 1, (int)gridDim.y);
    if (split >= splits) return;
    const int begin = split * p.chunk * S::kPerPage;               // in steps
    const int end = (split == splits - 1 ? count : (split + 1) * p.chunk) * S::kPerPage;

    RowState<D> st[C];
    Queries<D> q[C];
    const Cap cap = {p.cap_log2, p.cap_inverse};
    Slope slope[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        st[c].m = kNone;
        st[c].l = st[c].divisor = 0.0f;
#pragma unroll
        for (int m = 0; m < D / 16; ++m) st[c].o[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        q[c].load((const uint16_t *)p.q + (int64_t)(seq.start + i[c]) * p.q_token +
                      (int64_t)hq[c] * p.q_head,
                  mine[c], g);
        if constexpr (has_slopes(CHANGE)) {
            slope[c].set(p.slopes && mine[c] ? p.slopes[hq[c]] : 0.0f,
                         seq.length - seq.queries + i[c]);
        }
    }
    const int32_t *table = p.table + (int64_t)seq.index * p.width;
    const int64_t stride = (int64_t)p.kv_heads * Record<D>::kBytes;
    const uint8_t *cache = p.cache + (int64_t)head * Record<D>::kBytes;

    // 64 of this wave's steps at a time, one a lane: their numbers in the sequence, their
    // pages in the cache, and which are there
    int from = begin + wave, number = 0, phys = -1;
    uint64_t todo = 0;
    const auto look = [&]() {
        while (!todo && from < end) {
            const int e = from + kWaves * lane;
            from += kWaves * 64;
            number = page0 * S::kPerPage + e;
            phys = e < end ? table[number / S::kPerPage] : -1;
            todo = __builtin_amdgcn_ballot_w64(phys >= 0 && phys < p.pages);
        }
    };
    const auto next = [&](int &step) {
        const int at = __builtin_ctzll(todo);
        todo &= todo - 1;
        step = __builtin_amdgcn_readlane(number, at);
        return cache + (int64_t)__builtin_amdgcn_readlane(phys, at) * stride;
    };

    // Keys and values of one step are in registers at a time: the next one's keys are on
    // their way once this one's scores are there, its values once this one's are added.
    // (Two steps at a time, with less to hide them behind: 59 us as well.)
    u32x4 *const pieces = reinterpret_cast<u32x4 *>(&sh.o[wave][0][0]);
    look();
    typedef Keys<D, S::kTiles> K;
    K keys;
    Values<D, S::kTiles> values;
    u32x2 scales = {0, 0};
    int step = 0, biggest = kLeastScale;
    bool more = todo != 0;
    if (more) {
        const uint8_t *rec = next(step);
        scales = *reinterpret_cast<const u32x2 *>(rec + Record<D>::kScale);
        keys.template load<ONCE>(rec, step % S::kPerPage, lane);
        values.template load<ONCE>(rec, step % S::kPerPage, n, g);
        // (behind the loads: the queries have been on their way since before the page numbers)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < C; ++c) q[c].template settle<E>();
    }
    while (more) {
        const int t0 = step * S::kTokens;
        // whether some row does not see all of the step
        const bool masked = t0 < z.lo || t0 + S::kTokens > a.hi;
        // scales of the step's blocks (the bytes behind them are the page's others, or 0)
        const int before = step % S::kPerPage * 8 * S::kTiles;
        uint32_t ks = in_scalar(scales[0]) >> before, vs = in_scalar(scales[1]) >> before;
        if constexpr (S::kTiles < 4) ks &= 0xFFFFu, vs &= 0xFFFFu;
        if (masked) {
            const int lo = a.lo - t0, hi = min(z.hi - t0, S::kTokens);
            ks = settled_scales(ks, lo, hi);
            vs = settled_scales(vs, lo, hi);
        }
        const int km = largest_of(ks), vm = largest_of(vs);
        keys.store(pieces, lane);
        f32x4 s[C][S::kTiles];
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t) {
            const float f = relative(byte_of(ks, t), km, kUp<E>);
#pragma unroll
            for (int c = 0; c < C; ++c) s[c][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = 0; h < S::kChunks; ++h) {
                const u32x4 codes = pieces[K::place(16 * t + n, 4 * h + g)];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const u32x4 k = decode_eight<E>(codes[2 * x], codes[2 * x + 1], f, f);
#pragma unroll
                    for (int c = 0; c < C; ++c) s[c][t] = E::mfma16(k, q[c].q[h][x], s[c][t]);
                }
            }
        }
        look();
        more = todo != 0;
        const uint8_t *rec = nullptr;
        int following = 0;
        if (more) {
            rec = next(following);
            scales = *reinterpret_cast<const u32x2 *>(rec + Record<D>::kScale);
            keys.template load<ONCE>(rec, following % S::kPerPage, lane);
        }
        float scale = score_factor<E>(p.scale_log2, km);
        float offset = 0.0f;
        const auto all = [&](auto f) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int t = 0; t < S::kTiles; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k) s[c][t][k] = f(s[c][t][k], c, 16 * t + k);
        };
        if (CHANGE == Change::kCapped || (CHANGE == Change::kAny && cap.cap > 0.0f))
            cap.limit<CHANGE>(scale, offset,
                              [&](auto f) { all([&](float x, int, int) { return f(x); }); });
        if (CHANGE == Change::kSloped || (CHANGE == Change::kAny && p.slopes)) {
            float far[C];
#pragma unroll
            for (int c = 0; c < C; ++c) far[c] = slope[c].from(t0 + 4 * g);
            all([&](float x, int c, int j) { return slope[c](x * scale, far[c] - (float)j); });
            scale = 1.0f;
        }
        if (masked) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int lo = span[c].lo - t0 - 4 * g, hi = span[c].hi - t0 - 4 * g;
#pragma unroll
                for (int t = 0; t < S::kTiles; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int j = 16 * t + k;
                        s[c][t][k] = j >= lo && j < hi ? s[c][t][k] : -__builtin_inff();
                    }
            }
            values.clear(4 * g, a.lo - t0, z.hi - t0);
        }
        u32x4 w[C][S::kTiles / 2];
#pragma unroll
        for (int c = 0; c < C; ++c)
            weigh<E, D, CHANGE, FEW, S::kTiles>(st[c], s[c], w[c], scale, offset, paired, taken);
        if (vm > biggest) {
            const float f = relative(biggest, vm, 0);
            biggest = vm;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int m = 0; m < D / 16; ++m) st[c].o[m] *= f;
        }
        // ahead of the other waves' scores
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int u = 0; u < S::kTiles / 2; ++u) {
            const float f0 = relative(byte_of(vs, 2 * u), biggest, kUp<E>);
            const float f1 = relative(byte_of(vs, 2 * u + 1), biggest, kUp<E>);
#pragma unroll
            for (int h = 0; h < S::kChunks; ++h)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const u32x4 v = decode_eight<E>(values.v[2 * u][h][x],
                                                    values.v[2 * u + 1][h][x], f0, f1);
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        st[c].o[4 * h + x] = E::mfma16(v, w[c][u], st[c].o[4 * h + x]);
                }
        }
        __builtin_amdgcn_s_setprio(0);
        if (more) values.template load<ONCE>(rec, following % S::kPerPage, n, g);
        step = following;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const auto add = [](float x, float y) { return x + y; };
        const float l = across_rows(st[c].l, add), divisor = across_rows(st[c].divisor, add);
        if (g == 0) sh.ml[wave][16 * c + n] = f32x4{st[c].m, l, divisor, 0.0f};
#pragma unroll
        for (int h = 0; h < S::kChunks; ++h)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                sh.o[wave][16 * h + 4 * g + k][16 * c + n] =
                    f32x4{st[c].o[4 * h][k], st[c].o[4 * h + 1][k], st[c].o[4 * h + 2][k],
                          st[c].o[4 * h + 3][k]};
    }
    if (lane == 0) sh.scale[wave] = biggest;
    __syncthreads();

    // a thread for every four channels of a row, rows next to each other
    const int shift = valid > 1 ? 32 - __builtin_clz(valid - 1) : 0;   // rows, a power of two
    const auto write = [&](int r, int quad, const f32x4 &o, float top, float l, float divisor,
                           int scale) {
        const int rr = row0 + r;
        const int64_t at = (int64_t)(seq.start + rr / p.group) * (p.kv_heads * p.group) +
                           head * p.group + rr % p.group;
        *reinterpret_cast<u32x2 *>((typename E::T *)p.out + at * D + 4 * quad) =
            result<E>(o, divisor, scale);
        if (p.lse && quad == 0) p.lse[at] = log_sum(top, l);
    };
    typedef Part<D, kRows> P;
    float *part = p.part + (int64_t)unit * gridDim.y * P::kFloats;
    float *my = part + (int64_t)split * P::kFloats;
    int most = sh.scale[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) most = max(most, sh.scale[w]);
    for (int x = threadIdx.x; x < D / 4 << shift; x += kThreads) {
        const int r = x & ((1 << shift) - 1), quad = x >> shift;
        if (r >= valid) continue;
        // the waves' states in their order
        float top = sh.ml[0][r][0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sh.ml[w][r][0]);
        float l = 0.0f, divisor = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const f32x4 ml = sh.ml[w][r];
            const float f = __builtin_amdgcn_exp2f(ml[0] - top);
            l += ml[1] * f;
            divisor += ml[2] * f;
            f32x4 x = sh.o[w][quad][r];
            if (paired) x += sh.o[w][quad][r + 8];
            o += x * (f * relative(sh.scale[w], most, 0));
        }
        if (splits == 1) {
            write(r, quad, o, top, l, divisor, most);
        } else {
            // several splits: this one's state into the workspace
            if (quad == 0) {
                put(my + P::state(r), f32x2{top, l});
                put(my + P::state(r) + 2, f32x2{(float)most, divisor});
            }
            float *to = my + P::sums(valid, r, quad);
            put(to, f32x2{o[0], o[1]});
            put(to + 2, f32x2{o[2], o[3]});
        }
    }
    if (splits == 1) return;

    // the last split to get here joins them
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
        sh.last = last_of(p.tickets + (int64_t)unit * kTicketStride, splits);
    __syncthreads();
    if (!sh.last) return;
    for (int x = threadIdx.x; x < D / 4 << shift; x += kThreads) {
        const int r = x & ((1 << shift) - 1), quad = x >> shift;
        if (r >= valid) continue;
        const Joined j = join_parts<D, kRows>(part, splits, valid, r, quad);
        write(r, quad, j.o, j.top, j.l, j.divisor, j.scale);
    }
}

namespace {

template <typename E, int D, int C, bool FEW, bool ONCE>
void launch_c(const AttendParams &p, dim3 grid, hipStream_t s) {
    by_change(p, [&](auto kind) {
        hipLaunchKernelGGL((attend16_kernel<E, D, C, decltype(kind)::value, FEW, ONCE>), grid,
                           dim3(kThreads), 0, s, p);
    });
}

template <typename E, int D>
void launch_d(const AttendParams &p, int rows, bool few, bool once, dim3 grid, hipStream_t s) {
    if constexpr (D <= 128) {
        if (rows == 32) return launch_c<E, D, 2, false, false>(p, grid, s);
    }
    if (once) return launch_c<E, D, 1, true, true>(p, grid, s);
    if (few) return launch_c<E, D, 1, true, false>(p, grid, s);
    launch_c<E, D, 1, false, false>(p, grid, s);
}

template <typename E>
void launch_t(const AttendParams &p, int dim, int rows, bool few, bool once, dim3 grid,
              hipStream_t s) {
    if (dim == 64) launch_d<E, 64>(p, rows, few, once, grid, s);
    else if (dim == 128) launch_d<E, 128>(p, rows, few, once, grid, s);
    else launch_d<E, 256>(p, rows, few, once, grid, s);
}

}  // namespace

void launch_attend16(const AttendParams &p, int type, int dim, int rows, bool few, bool once,
                     dim3 grid, hipStream_t s) {
    if (type == LCE_FLOAT16) launch_t<F16>(p, dim, rows, few, once, grid, s);
    else launch_t<Bf16>(p, dim, rows, few, once, grid, s);
}

}  // namespace kv8
}  // namespace lce
