// Attention over the 4-bit cache, 16 or 32 query rows a tile: single tokens, a few
// tokens, short prompts, and lists of pages.
#include "kv4_attend.hpp"

namespace lce {
namespace kv4 {
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

// One page of one head as a wave's 64 lanes hold it.  Lane (n, g), n = lane %
// 16, g = lane / 16: the key codes of tokens 16t + n, 16 bytes of them for each
// 128 channels (the first operand of a 16x16x128 product: 32 channels in a row),
// and the value codes of tokens 16t + 4g + i for the D/16 channels from
// D/16 * n on.
template <int D>
struct Keys {
    static constexpr int kChunks = D < 128 ? 1 : D / 128;
    u32x4 k[4][kChunks];
    uint32_t scale[kChunks];   // byte t: scale of tokens 16t + n

    template <bool ONCE>
    __device__ __forceinline__ void load(const uint8_t *rec, int n, int g) {
        // a head of 64 channels fills half of the product's 128: the other half
        // repeats them, against another piece of the queries
        const int kg = D < 128 ? g % 2 : g;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
                k[t][c] = fetch<ONCE, u32x4>(rec + (16 * t + n) * (D / 2) + 64 * c +
                                                           16 * kg);
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            scale[c] = fetch<ONCE, uint32_t>(rec + Record<D>::kKeyScale +
                                                           (n * (D / 32) + 4 * c + kg) * 4);
    }
};

template <int D>
struct Values {
    uint32_t v[4][D / 32];
    u32x4 scale;               // byte i of word t: scale of token 16t + 4g + i

    template <bool ONCE>
    __device__ __forceinline__ void load(const uint8_t *rec, int n, int g) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint8_t *at = rec + Record<D>::kValue + ((4 * t + g) * 16 + n) * (D / 8);
            if constexpr (D == 64) {
                const u32x2 w = fetch<ONCE, u32x2>(at);
                v[t][0] = w[0], v[t][1] = w[1];
            } else {
#pragma unroll
                for (int j = 0; j < D / 128; ++j) {
                    const u32x4 w = fetch<ONCE, u32x4>(at + 16 * j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[t][4 * j + i] = w[i];
                }
            }
        }
        // channels D/16 * n lie in group n * D / 512
        scale = fetch<ONCE, u32x4>(rec + Record<D>::kValueScale +
                                                 (n * D / 512) * 64 + 16 * g);
    }
};

// Queries of 16 rows as second operands: lane (n, g) holds, of row n, channels
// 16g .. +15 and 64 + 16g .. +15 of each 128 (the order of an 8-bit operand),
// in pieces.
template <typename E, int D>
struct Queries {
    static constexpr int kChunks = Keys<D>::kChunks;
    // products per 128 channels (per head where D = 64: there one product takes
    // two pieces, in its two halves)
    static constexpr int kSteps = D < 128 ? (E::kPieces + 1) / 2 : E::kPieces;
    i32x8 piece[kSteps][kChunks];
    uint32_t scale[kChunks];   // byte st: the scale of the lane's group in product st
};

// The same channels as they come from memory: on their way while the page
// numbers are, and made into pieces while the first page is.
template <int D>
struct RawQueries {
    static constexpr int kHalves = D < 128 ? 1 : 2;
    u32x4 w[Keys<D>::kChunks][kHalves][2];

    __device__ __forceinline__ void load(const void *row, bool valid, int g) {
#pragma unroll
        for (int c = 0; c < Keys<D>::kChunks; ++c)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                w[c][h][0] = w[c][h][1] = u32x4{0, 0, 0, 0};
                if (valid) {
                    const u32x4 *at = reinterpret_cast<const u32x4 *>(
                        static_cast<const uint16_t *>(row) + 128 * c + 64 * h + 16 * g);
                    w[c][h][0] = at[0], w[c][h][1] = at[1];
                }
            }
    }
};

// Lane (n, g) holds half of channel group g / 2, and of group 2 + g / 2 in its second
// half, and gives the products the scale of group g: heads of 64 channels, of which
// a product takes two pieces, that of group g % 2 for piece g / 2.
template <typename E, int D>
__device__ __forceinline__ void make_pieces(Queries<E, D> &q, const RawQueries<D> &raw, int g) {
    constexpr int kChunks = Keys<D>::kChunks, kHalves = RawQueries<D>::kHalves;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        uint32_t bytes[E::kPieces][kHalves][4];
        f32x2 tops[kHalves];
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            float x[16];
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t w = raw.w[c][h][i / 4][i % 4];
                bits = max(bits, max(w & 0x7FFFu, w >> 16 & 0x7FFFu));
                const typename E::T2 pair = bits_as<typename E::T2>(w);
                x[2 * i] = (float)pair[0];
                x[2 * i + 1] = (float)pair[1];
            }
            const uint32_t own = bits_as<uint32_t>(top_of<E>(bits));
            const auto a = __builtin_amdgcn_permlane16_swap(own, own, false, false);
            const float top =
                fmaxf(bits_as<float>((uint32_t)a[0]), bits_as<float>((uint32_t)a[1]));
            tops[h] = both_halves(top);
            const float up = group_scale<E>(top).up;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = x[4 * i + j] * up;
#pragma unroll
                for (int p = 0; p < E::kPieces; ++p) bytes[p][h][i] = next_piece(y);
            }
        }
        if constexpr (D < 128) {
            const uint32_t scales = group_scale<E>(g % 2 ? tops[0][1] : tops[0][0]).bytes;
            q.scale[c] = 0;
#pragma unroll
            for (int st = 0; st < Queries<E, D>::kSteps; ++st) {
                const int p0 = 2 * st, p1 = 2 * st + 1 < E::kPieces ? 2 * st + 1 : p0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    q.piece[st][c][i] = (int)bytes[p0][0][i];
                    q.piece[st][c][4 + i] = p1 == p0 ? 0 : (int)bytes[p1][0][i];
                }
                q.scale[c] |= (scales >> (g < 2 ? 8 * p0 : 8 * p1) & 255u) << (8 * st);
            }
        } else {
            const f32x2 top = tops[g < 2 ? 0 : kHalves - 1];
            q.scale[c] = group_scale<E>(g % 2 ? top[1] : top[0]).bytes;
#pragma unroll
            for (int p = 0; p < E::kPieces; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    q.piece[p][c][i] = (int)bytes[p][0][i];
                    q.piece[p][c][4 + i] = (int)bytes[p][kHalves - 1][i];
                }
        }
    }
}

// A chunk's product of step ST, and those of the steps after it.
template <typename E, int D, int T, int ST>
__device__ __forceinline__ f32x4 multiply(const i32x8 &k, uint32_t scale, const Queries<E, D> &q,
                                          int c, f32x4 s) {
    if constexpr (ST < Queries<E, D>::kSteps) {
        s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q.piece[ST][c], s, 4, 0, T,
                                                             (int)scale, ST, (int)q.scale[c]);
        return multiply<E, D, T, ST + 1>(k, scale, q, c, s);
    }
    return s;
}

// Scores of a page: s[t][i] of lane (n, g) is row n against token 16t + 4g + i.
template <typename E, int D, int T>
__device__ __forceinline__ f32x4 scores(const Keys<D> &r, const Queries<E, D> &q) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < Keys<D>::kChunks; ++c) {
        const u32x4 k = r.k[T][c];
        s = multiply<E, D, T, 0>(i32x8{(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0},
                                 r.scale[c], q, c, s);
    }
    return s;
}

// A row's state: running maximum of scaled scores (log2), this lane's share of
// the sum, and the sums of weighted values: o[m][i] of lane (n, g) is row n,
// channel D/16 * (4g + i) + m.
template <int D>
struct RowState {
    float m, l;
    f32x4 o[D / 16];
};

// The values of token pairs: byte B of a token's codes holds its channels 2B
// and 2B+1; a product wants two tokens of one channel side by side.
template <typename E, int D, int TAU, int B, bool SAT>
__device__ __forceinline__ void decode_values(const Values<D> &r, uint32_t (&even)[2],
                                              uint32_t (&odd)[2]) {
    constexpr int G = D / 32;
    // the bits beside the exponent's do not count: a shift makes a scale's byte one
    const uint32_t w = r.scale[TAU];
    const uint32_t x0 = decode_pair<E, B % 4, SAT>(r.v[TAU][B / 4], bits_as<float>(w << 23));
    const uint32_t x1 =
        decode_pair<E, (G + B) % 4, SAT>(r.v[TAU][(G + B) / 4], bits_as<float>(w << 15));
    const uint32_t x2 =
        decode_pair<E, (2 * G + B) % 4, SAT>(r.v[TAU][(2 * G + B) / 4], bits_as<float>(w << 7));
    const uint32_t x3 =
        decode_pair<E, (3 * G + B) % 4, SAT>(r.v[TAU][(3 * G + B) / 4], bits_as<float>(w >> 1));
    even[0] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
    odd[0] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
    even[1] = __builtin_amdgcn_perm(x3, x2, 0x05040100u);
    odd[1] = __builtin_amdgcn_perm(x3, x2, 0x07060302u);
}

template <typename E, int D, int C, int U, int B, bool SAT>
__device__ __forceinline__ void add_values(RowState<D> (&st)[C], const Values<D> &r,
                                           const u32x4 (&p)[C][2]) {
    if constexpr (B < D / 32) {
        uint32_t e0[2], o0[2], e1[2], o1[2];
        decode_values<E, D, 2 * U, B, SAT>(r, e0, o0);
        decode_values<E, D, 2 * U + 1, B, SAT>(r, e1, o1);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            st[c].o[2 * B] =
                E::mfma16(u32x4{e0[0], e0[1], e1[0], e1[1]}, p[c][U], st[c].o[2 * B]);
            st[c].o[2 * B + 1] =
                E::mfma16(u32x4{o0[0], o0[1], o1[0], o1[1]}, p[c][U], st[c].o[2 * B + 1]);
        }
        add_values<E, D, C, U, B + 1, SAT>(st, r, p);
    }
}

// Hides the tokens outside [lo, hi) (this row's visible ones, counted from the lane's
// first: 4g on the page, so that constants are compared with two registers).
__device__ __forceinline__ void hide(f32x4 (&s)[4], int lo, int hi) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = 16 * t + i;
            s[t][i] = j >= lo && j < hi ? s[t][i] : -__builtin_inff();
        }
}

// Takes the values past the type's range out of a page (their scale to almost nothing);
// whether some lane had one.
template <typename E, int D>
__device__ __forceinline__ bool take_past_range(Values<D> &r) {
    if constexpr (!E::kSaturates) return false;
    const uint32_t any = past_float16(r.scale[0]) | past_float16(r.scale[1]) |
                         past_float16(r.scale[2]) | past_float16(r.scale[3]);
    const bool past = __builtin_amdgcn_ballot_w64(any != 0) != 0;
    if (__builtin_expect(past, 0)) {
#pragma unroll
        for (int t = 0; t < 4; ++t) r.scale[t] &= ~whole_bytes(past_float16(r.scale[t]));
    }
    return past;
}

// A page's scores into the rows' maximum and sum; its weights, ready to be
// multiplied.
template <typename E, int D>
__device__ __forceinline__ void weigh(RowState<D> &st, f32x4 (&s)[4], u32x4 (&p)[2], float c) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
    top *= c;
    // (Of large maxima, the difference is exact where a sum is not.  Each row goes by
    // its own maximum, so that no bit of it depends on the rows beside it.)
    if (__builtin_amdgcn_ballot_w64(top - st.m > kLag + E::kLift)) {
        const float high = across_rows(top, [](float a, float b) { return fmaxf(a, b); });
        const float all = high - st.m > kLag + E::kLift ? high - E::kLift : st.m;
        const float f = __builtin_amdgcn_exp2f(st.m - all);
        st.m = all;
        st.l *= f;
#pragma unroll
        for (int m = 0; m < D / 16; ++m) st.o[m] *= f;
    }
    // The fused product below differs from the rounded one that the maximum is; where
    // that could show (scores past kLarge), round the scores' products too.
    const bool large = __builtin_fabsf(st.m) > kLarge;
    if (__builtin_amdgcn_ballot_w64(large)) {
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] = large ? s[t] * c : s[t];
        c = large ? 1.0f : c;
    }
    // a page's weights are summed by themselves: a long sequence's many small ones would
    // be rounded one by one to the last place of a large sum
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], c, -st.m));
            sum += w[i];
        }
        p[t / 2][t % 2 * 2] = pack_pair<E>(w[0], w[1]);
        p[t / 2][t % 2 * 2 + 1] = pack_pair<E>(w[2], w[3]);
    }
    st.l += sum;
}

// The waves' states, where they are joined: sums four channels at a time, rows next
// to each other.
template <int D, int C>
struct Shared {
    f32x4 o[kWaves][D / 4][16 * C];
    f32x2 ml[kWaves][16 * C];
    int last;
};

}  // namespace

// Grid (tiles * kv_heads, splits), four waves.  A tile is C times 16 rows of one head
// of the cache: rows are the queries of one sequence times the heads that share
// the cache head, in that order (with LIST, those of one token).  The waves take
// the pages of their workgroup's split in turn, each with all rows, and
// join their states at the end; the last split of a tile to finish joins all of
// them, in the order of the splits, so that results do not depend on timing.
//
// Keys are the first operand and queries the second, so that a lane's scores
// belong to one row and the weights leave the softmax as the second operand of
// the product with the values; no weight and no score crosses lanes.
//
// Bound by memory where a call reads much, by the latencies in a row (launch,
// lengths, table, a page, the states out, the ticket, the states in) where it does
// not.  Measured, us: 64 sequences of up to 8192 tokens, 64 heads of 128 on 8, bfloat16
// (238 MB) 51.2, 4.6 TB/s with the launch; one sequence of 20001, 32 heads on 8
// (22 MB) 11.9, of which the joining of the splits takes 3; 128 lists of 64 pages
// (61 MB) 16.1.  Loads of a page's keys and values are 16 bytes a lane, and one page
// is on its way while another is worked on: 12 waves of a CU hide the rest.  What
// float16's range costs (values past it, looked for in every page): up to 2 %, in tiles
// of 32 rows 5 %.
template <typename E, int D, bool LIST, int C, bool ONCE>
__global__ __launch_bounds__(kThreads, D <= 128 && C == 1 ? 3 : 2) void attend16_kernel(
    AttendParams p) {
    constexpr int kRows = 16 * C;
    __shared__ Shared<D, C> sh;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the eight XCDs in turn, and where the grid is a multiple of eight
    // wide all splits of a tile would go to one.  Where the heads do not spread a long
    // sequence over the XCDs, its tiles are moved on by one a split (32 sequences of up
    // to 53109 tokens, 16 heads on one: 47 -> 33 us).
    const int split = blockIdx.y;
    int unit = blockIdx.x;
    if (!LIST && p.turn) {
        unit += split % 8;
        if (unit >= p.turn) unit -= p.turn;
    }
    const int head = unit % p.kv_heads, slot = unit / p.kv_heads;

    // the tile: rows of a sequence, or of a token
    Sequence seq;
    int tile, token = 0;
    if constexpr (LIST) {
        const int per = (p.group + kRows - 1) / kRows;
        token = slot / per;
        tile = slot % per;
        seq = find_sequence(p.q_start, p.lengths, p.seqs, p.tokens, p.width, token,
                            [](int s, int) { return (int64_t)s; });
        if (seq.index < 0 || token - seq.start >= seq.queries) return;
    } else {
        // a sequence's tiles begin at floor(rows before it / kRows) + its index:
        // at most one more than it needs, and none shared
        const auto first = [&](int s, int b) { return (int64_t)s * p.group / kRows + b; };
        seq = find_sequence(p.q_start, p.lengths, p.seqs, p.tokens, p.width, slot, first);
        if (seq.index < 0) return;
        tile = (int)(slot - first(seq.start, seq.index));
    }
    const int rows = LIST ? p.group : seq.queries * p.group;
    const int row0 = tile * kRows;
    if (row0 >= rows) return;
    const int valid = min(rows - row0, kRows);
    const int base = LIST ? (token - seq.start) * p.group : 0;   // in rows of the sequence
    // this lane's row of each sixteen
    int i[C], hq[C];
    bool mine[C];
    Span span[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int row = base + row0 + 16 * c + n;
        i[c] = row / p.group, hq[c] = head * p.group + row % p.group;
        mine[c] = 16 * c + n < valid;
        span[c] = visible(seq, i[c], p.causal, p.window);
    }
    // spans move up with the rows: the tile's first and last row bound them
    const Span a = visible(seq, (base + row0) / p.group, p.causal, p.window);
    const Span z = visible(seq, (base + row0 + valid - 1) / p.group, p.causal, p.window);

    // this workgroup's share of the pages (LIST: of the list's entries)
    const int page0 = LIST ? 0 : a.lo / kPage;
    const int count = LIST ? p.list : z.hi > a.lo ? (z.hi + kPage - 1) / kPage - page0 : 0;
    const int splits = clampi((count + p.chunk - 1) / p.chunk, 1, (int)gridDim.y);
    if (split >= splits) return;
    const int begin = split * p.chunk;
    const int end = split == splits - 1 ? count : begin + p.chunk;

    RowState<D> st[C];
    RawQueries<D> raw[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        st[c].m = kNone;
        st[c].l = 0.0f;
#pragma unroll
        for (int m = 0; m < D / 16; ++m) st[c].o[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        raw[c].load((const typename E::T *)p.q + (int64_t)(seq.start + i[c]) * p.q_token +
                        (int64_t)hq[c] * p.q_head,
                    mine[c], g);
    }
    const int32_t *named =
        LIST ? p.named + ((int64_t)(seq.start + base / p.group) * p.kv_heads + head) * p.list
             : nullptr;
    const int32_t *table = p.table + (int64_t)seq.index * p.width;
    const int64_t stride = (int64_t)p.kv_heads * Record<D>::kBytes;
    const uint8_t *cache = p.cache + (int64_t)head * Record<D>::kBytes;
    const int last_page = (z.hi + kPage - 1) / kPage;

    // 64 of this wave's pages at a time, one a lane: their numbers in the
    // sequence and in the cache, and which are there
    int from = begin + wave, page = -1, phys = -1;
    uint64_t todo = 0;
    const auto fetch = [&]() {
        while (!todo && from < end) {
            const int e = from + kWaves * lane;
            from += kWaves * 64;
            page = phys = -1;
            if (e < end) {
                page = LIST ? named[e] : page0 + e;
                if (page >= 0 && page < last_page) phys = table[page];
            }
            todo = __builtin_amdgcn_ballot_w64(phys >= 0 && phys < p.pages);
        }
    };
    const auto next = [&](int &number) {
        const int at = __builtin_ctzll(todo);
        todo &= todo - 1;
        number = __builtin_amdgcn_readlane(page, at);
        return cache + (int64_t)__builtin_amdgcn_readlane(phys, at) * stride;
    };

    // Keys and values of one page are in registers at a time: the next page's
    // keys are on their way once this page's weights are there, its values once
    // this page's are added.
    fetch();
    Keys<D> keys;
    Values<D> values;
    int number = 0;
    const uint8_t *now = nullptr;
    const bool any = todo != 0;
    if (any) {
        now = next(number);
        keys.template load<ONCE>(now, n, g);
        values.template load<ONCE>(now, n, g);
    }
    const auto settle = [&](Values<D> &v, int t0) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
            v.scale[t] = settled(v.scale[t], 16 * t, a.lo - t0 - 4 * g, z.hi - t0 - 4 * g);
    };
    Queries<E, D> q[C];
#pragma unroll
    for (int c = 0; c < C; ++c) make_pieces<E, D>(q[c], raw[c], g);
    bool more = any;
    while (more) {
        const int t0 = number * kPage;
        const bool masked = t0 < z.lo || t0 + kPage > a.hi;
        f32x4 s[C][4];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            s[c][0] = scores<E, D, 0>(keys, q[c]);
            s[c][1] = scores<E, D, 1>(keys, q[c]);
            s[c][2] = scores<E, D, 2>(keys, q[c]);
            s[c][3] = scores<E, D, 3>(keys, q[c]);
        }
        fetch();
        more = todo != 0;
        const uint8_t *rec = nullptr;
        if (more) rec = next(number);
        if (masked) {
#pragma unroll
            for (int c = 0; c < C; ++c) hide(s[c], span[c].lo - t0 - 4 * g, span[c].hi - t0 - 4 * g);
            settle(values, t0);
        }
        u32x4 w[C][2];
#pragma unroll
        for (int c = 0; c < C; ++c) weigh<E, D>(st[c], s[c], w[c], p.scale_log2);
        if (more) keys.template load<ONCE>(rec, n, g);
        const bool past = take_past_range<E, D>(values);
        // ahead of the other waves' scores: 1 to 3 % (heads of 256, 128 rows on 65536
        // tokens: 386 -> 376 us)
        __builtin_amdgcn_s_setprio(1);
        add_values<E, D, C, 0, 0, false>(st, values, w);
        add_values<E, D, C, 1, 0, false>(st, values, w);
        __builtin_amdgcn_s_setprio(0);
        // the values past the range from memory once more, and saturated: a second set of
        // them here would cost registers everywhere
        if (__builtin_expect(past, 0)) {
            values.template load<ONCE>(now, n, g);
            if (masked) settle(values, t0);
#pragma unroll
            for (int t = 0; t < 4; ++t) values.scale[t] &= whole_bytes(past_float16(values.scale[t]));
            add_values<E, D, C, 0, 0, E::kSaturates>(st, values, w);
            add_values<E, D, C, 1, 0, E::kSaturates>(st, values, w);
        }
        if (more) values.template load<ONCE>(rec, n, g);
        now = rec;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const float l = across_rows(st[c].l, [](float x, float y) { return x + y; });
        if (g == 0) sh.ml[wave][16 * c + n] = f32x2{st[c].m, l};
        // quad (j, m / 4, g): channels D/16 * (4g + j) + m .. m + 3
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int m = 0; m < D / 16; m += 4)
                sh.o[wave][(j * (D / 64) + m / 4) * 4 + g][16 * c + n] =
                    f32x4{st[c].o[m][j], st[c].o[m + 1][j], st[c].o[m + 2][j], st[c].o[m + 3][j]};
    }
    __syncthreads();

    // a thread for every four channels of a row, rows next to each other
    const int shift = valid > 1 ? 32 - __builtin_clz(valid - 1) : 0;   // rows, a power of two
    const auto write = [&](int r, int quad, const f32x4 &o, float top, float l) {
        const int c = D / 16 * (4 * (quad % 4) + quad / 4 / (D / 64)) + quad / 4 % (D / 64) * 4;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const int rr = base + row0 + r;
        const int64_t at = (int64_t)(seq.start + rr / p.group) * (p.kv_heads * p.group) +
                           head * p.group + rr % p.group;
        *reinterpret_cast<u32x2 *>((typename E::T *)p.out + at * D + c) =
            u32x2{pack_result<E>(o[0] * inv, o[1] * inv),
                  pack_result<E>(o[2] * inv, o[3] * inv)};
        if (p.lse && quad == 0)
            p.lse[at] = l == 0.0f ? -__builtin_inff()
                                  : (top + __builtin_log2f(l)) * 0.69314718055994531f;
    };
    typedef Part<D, kRows> P;
    float *part = p.part + (int64_t)unit * gridDim.y * P::kFloats;
    float *my = part + (int64_t)split * P::kFloats;
    for (int x = threadIdx.x; x < D / 4 << shift; x += kThreads) {
        const int r = x & ((1 << shift) - 1), quad = x >> shift;
        if (r >= valid) continue;
        // the waves' states in their order
        float top = sh.ml[0][r][0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sh.ml[w][r][0]);
        float l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const f32x2 ml = sh.ml[w][r];
            const float f = __builtin_amdgcn_exp2f(ml[0] - top);
            l += ml[1] * f;
            o += sh.o[w][quad][r] * f;
        }
        if (splits == 1) {
            write(r, quad, o, top, l);
        } else {
            // several splits: this one's state into the workspace
            if (quad == 0) put(my + P::state(r), f32x2{top, l});
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
        float top, l;
        const f32x4 o = join_splits<D, kRows>(part, splits, valid, r, quad, top, l);
        write(r, quad, o, top, l);
    }
}

namespace {

template <typename E, int D, int C, bool ONCE>
void launch_c(const AttendParams &p, dim3 grid, hipStream_t s) {
    if constexpr (C == 1) {
        if (p.named) {
            hipLaunchKernelGGL((attend16_kernel<E, D, true, 1, ONCE>), grid, dim3(kThreads), 0, s, p);
            return;
        }
    }
    hipLaunchKernelGGL((attend16_kernel<E, D, false, C, ONCE>), grid, dim3(kThreads), 0, s, p);
}

template <typename E, int D>
void launch_d(const AttendParams &p, int rows, bool once, dim3 grid, hipStream_t s) {
    // 32 rows of 128 channels in float16, or of 256, have more state than registers
    if constexpr (D * E::kPieces <= 256) {
        if (rows == 32) return launch_c<E, D, 2, false>(p, grid, s);
    }
    if constexpr (D == 128) {
        if (once) return launch_c<E, D, 1, true>(p, grid, s);
    }
    launch_c<E, D, 1, false>(p, grid, s);
}

template <typename E>
void launch_t(const AttendParams &p, int dim, int rows, bool once, dim3 grid, hipStream_t s) {
    if (dim == 64) launch_d<E, 64>(p, rows, once, grid, s);
    else if (dim == 128) launch_d<E, 128>(p, rows, once, grid, s);
    else launch_d<E, 256>(p, rows, once, grid, s);
}

}  // namespace

void launch_attend16(const AttendParams &p, int type, int dim, int rows, bool once, dim3 grid,
                     hipStream_t s) {
    if (type == LCE_FLOAT16) launch_t<F16>(p, dim, rows, once, grid, s);
    else launch_t<Bf16>(p, dim, rows, once, grid, s);
}

}  // namespace kv4
}  // namespace lce
