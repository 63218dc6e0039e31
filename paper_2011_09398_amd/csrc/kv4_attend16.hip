// Attention over the 4-bit cache, 16 query rows a tile: single tokens, a few
// tokens, and lists of pages.
#include "kv4_attend.hpp"

namespace lce {
namespace kv4 {
namespace {

constexpr int kWaves = kThreads / 64;
constexpr int kRows = 16;

// One page of one head as a wave's 64 lanes hold it.  Lane (n, g), n = lane %
// 16, g = lane / 16: the key codes of tokens 16t + n, 16 bytes of them for each
// 128 channels (the first operand of a 16x16x128 product: 32 channels in a row),
// and the value codes of tokens 16t + 4g + i for the D/16 channels from
// D/16 * n on.
template <int D>
struct PageRegs {
    static constexpr int kChunks = D < 128 ? 1 : D / 128;
    u32x4 k[4][kChunks];
    uint32_t v[4][D / 32];
    uint32_t ks[kChunks];   // byte t: scale of tokens 16t + n
    u32x4 vs;               // byte i of word t: scale of token 16t + 4g + i
};

template <int D>
__device__ __forceinline__ void load_page(PageRegs<D> &r, const uint8_t *rec, int n, int g) {
    typedef PageRegs<D> P;
    // a head of 64 channels fills half of the product's 128: the other half
    // repeats them, against another piece of the queries
    const int kg = D < 128 ? g % 2 : g;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int c = 0; c < P::kChunks; ++c)
            r.k[t][c] = *reinterpret_cast<const u32x4 *>(rec + (16 * t + n) * (D / 2) + 64 * c +
                                                         16 * kg);
#pragma unroll
    for (int c = 0; c < P::kChunks; ++c)
        r.ks[c] = *reinterpret_cast<const uint32_t *>(rec + Record<D>::kKeyScale +
                                                      (n * (D / 32) + 4 * c + kg) * 4);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint8_t *at = rec + Record<D>::kValue + ((4 * t + g) * 16 + n) * (D / 8);
        if constexpr (D == 64) {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(at);
            r.v[t][0] = w[0], r.v[t][1] = w[1];
        } else {
#pragma unroll
            for (int j = 0; j < D / 128; ++j) {
                const u32x4 w = reinterpret_cast<const u32x4 *>(at)[j];
#pragma unroll
                for (int i = 0; i < 4; ++i) r.v[t][4 * j + i] = w[i];
            }
        }
    }
    // channels D/16 * n lie in group n * D / 512
    r.vs = *reinterpret_cast<const u32x4 *>(rec + Record<D>::kValueScale + (n * D / 512) * 64 +
                                            16 * g);
}

// Queries of 16 rows as second operands: lane (n, g) holds, of row n, channels
// 16g .. +15 and 64 + 16g .. +15 of each 128 (the order of an 8-bit operand),
// in pieces.
template <typename E, int D>
struct Queries {
    static constexpr int kChunks = PageRegs<D>::kChunks;
    // products per 128 channels (per head where D = 64: there one product takes
    // two pieces, in its two halves)
    static constexpr int kSteps = D < 128 ? (E::kPieces + 1) / 2 : E::kPieces;
    i32x8 piece[kSteps][kChunks];
    uint32_t scale[kSteps];
};

template <typename E, int D>
__device__ __forceinline__ void load_queries(Queries<E, D> &q, const typename E::T *row, bool valid,
                                             int g) {
    constexpr int kChunks = PageRegs<D>::kChunks, kHalves = D < 128 ? 1 : 2;
    float x[kChunks][kHalves][16];
    float top = 0.0f;
    bool odd = false;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            u32x4 w[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
            if (valid) {
                const u32x4 *at = reinterpret_cast<const u32x4 *>(row + 128 * c + 64 * h + 16 * g);
                w[0] = at[0], w[1] = at[1];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t word = w[i / 8][i % 8 / 2];
                const typename E::T2 pair = bits_as<typename E::T2>(word);
                x[c][h][i] = (float)pair[i % 2];
                odd |= !(__builtin_fabsf(x[c][h][i]) < __builtin_inff());
                top = fmaxf(top, __builtin_fabsf(x[c][h][i]));
            }
        }
    if (odd) top = __builtin_inff();
    top = across_rows(top, [](float a, float b) { return fmaxf(a, b); });
    const RowScale s = row_scale(top);
    uint32_t bytes[E::kPieces][kChunks][kHalves][4];
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = x[c][h][4 * i + j] * s.up;
#pragma unroll
                for (int p = 0; p < E::kPieces; ++p) bytes[p][c][h][i] = next_piece(y);
            }
    // the scale of piece p: 16^-p
    const auto scale = [&](int p) { return s.byte == 255u ? 255u : s.byte - 4u * p; };
    if constexpr (D < 128) {
#pragma unroll
        for (int st = 0; st < Queries<E, D>::kSteps; ++st) {
            const int p0 = 2 * st, p1 = 2 * st + 1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                q.piece[st][0][i] = (int)bytes[p0][0][0][i];
                q.piece[st][0][4 + i] = p1 < E::kPieces ? (int)bytes[p1 < E::kPieces ? p1 : 0][0][0][i] : 0;
            }
            // scales go by the product's groups of 32: its second half is piece p1
            q.scale[st] = g < 2 ? scale(p0) : scale(p1 < E::kPieces ? p1 : p0);
        }
    } else {
#pragma unroll
        for (int p = 0; p < E::kPieces; ++p) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    q.piece[p][c][i] = (int)bytes[p][c][0][i];
                    q.piece[p][c][4 + i] = (int)bytes[p][c][kHalves - 1][i];
                }
            q.scale[p] = scale(p);
        }
    }
}

// Scores of a page: s[t][i] of lane (n, g) is row n against token 16t + 4g + i.
template <typename E, int D, int T>
__device__ __forceinline__ f32x4 scores(const PageRegs<D> &r, const Queries<E, D> &q) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < PageRegs<D>::kChunks; ++c) {
        const u32x4 k = r.k[T][c];
        const i32x8 a = {(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < Queries<E, D>::kSteps; ++st)
            s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.piece[st][c], s, 4, 0, T,
                                                                 (int)r.ks[c], 0, (int)q.scale[st]);
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
template <typename E, int D, int TAU, int B>
__device__ __forceinline__ void decode_values(const PageRegs<D> &r, const float (&scale)[4],
                                              uint32_t (&even)[2], uint32_t (&odd)[2]) {
    constexpr int G = D / 32;
    uint32_t x[4];
#define LCE_KV4_TOKEN(I) \
    x[I] = decode_pair<E, (I * G + B) % 4>(r.v[TAU][(I * G + B) / 4], scale[I])
    LCE_KV4_TOKEN(0);
    LCE_KV4_TOKEN(1);
    LCE_KV4_TOKEN(2);
    LCE_KV4_TOKEN(3);
#undef LCE_KV4_TOKEN
    even[0] = __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
    odd[0] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
    even[1] = __builtin_amdgcn_perm(x[3], x[2], 0x05040100u);
    odd[1] = __builtin_amdgcn_perm(x[3], x[2], 0x07060302u);
}

template <typename E, int D, int U, int B>
__device__ __forceinline__ void add_values(RowState<D> &st, const PageRegs<D> &r,
                                           const float (&s0)[4], const float (&s1)[4],
                                           const u32x4 &p) {
    if constexpr (B < D / 32) {
        uint32_t e0[2], o0[2], e1[2], o1[2];
        decode_values<E, D, 2 * U, B>(r, s0, e0, o0);
        decode_values<E, D, 2 * U + 1, B>(r, s1, e1, o1);
        st.o[2 * B] = E::mfma16(u32x4{e0[0], e0[1], e1[0], e1[1]}, p, st.o[2 * B]);
        st.o[2 * B + 1] = E::mfma16(u32x4{o0[0], o0[1], o1[0], o1[1]}, p, st.o[2 * B + 1]);
        add_values<E, D, U, B + 1>(st, r, s0, s1, p);
    }
}

// One page into the rows' state.  MASK: some row does not see some token (lo,
// hi: this row's visible tokens, counted from the page's first).
template <typename E, int D, bool MASK>
__device__ __forceinline__ void attend_page(RowState<D> &st, const PageRegs<D> &r,
                                            const Queries<E, D> &q, float c, int lo, int hi,
                                            int g) {
    f32x4 s[4] = {scores<E, D, 0>(r, q), scores<E, D, 1>(r, q), scores<E, D, 2>(r, q),
                  scores<E, D, 3>(r, q)};
    float top = -__builtin_inff();
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (MASK) {
                const int j = 16 * t + 4 * g + i;
                s[t][i] = j >= lo && j < hi ? s[t][i] : -__builtin_inff();
            }
            top = fmaxf(top, s[t][i]);
        }
    top *= c;
    // The maximum that weights are taken against follows the true one only when
    // that has passed it by 2^8: weights up to 256 cost no precision, and most
    // pages then need neither the exchange between lanes nor the rescaling.
    if (__builtin_amdgcn_ballot_w64(top > st.m + 8.0f)) {
        const float all =
            fmaxf(st.m, across_rows(top, [](float a, float b) { return fmaxf(a, b); }));
        const float f = __builtin_amdgcn_exp2f(st.m - all);
        st.m = all;
        st.l *= f;
#pragma unroll
        for (int m = 0; m < D / 16; ++m) st.o[m] *= f;
    }
    u32x4 p[2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], c, -st.m));
            st.l += w[i];
        }
        p[t / 2][t % 2 * 2] = pack_pair<E>(w[0], w[1]);
        p[t / 2][t % 2 * 2 + 1] = pack_pair<E>(w[2], w[3]);
    }
    float scale[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (MASK)
                scale[t][i] = scale_of(min(r.vs[t] >> (8 * i) & 255u, E::kMaxScale));
            else   // the bits beside the exponent's do not count
                scale[t][i] = bits_as<float>(i < 3 ? r.vs[t] << (23 - 8 * i) : r.vs[t] >> 1);
        }
    add_values<E, D, 0, 0>(st, r, scale[0], scale[1], p[0]);
    add_values<E, D, 1, 0>(st, r, scale[2], scale[3], p[1]);
}

// Joins another state of the same rows into this one.
template <int D>
__device__ __forceinline__ void join(RowState<D> &a, float m, float l, const f32x4 (&o)[D / 16]) {
    const float all = fmaxf(a.m, m);
    const float fa = __builtin_amdgcn_exp2f(a.m - all), fb = __builtin_amdgcn_exp2f(m - all);
    a.m = all;
    a.l = a.l * fa + l * fb;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) a.o[i] = a.o[i] * fa + o[i] * fb;
}

template <typename E, int D>
struct Shared {
    float o[2][D / 16 * 4][64];
    float m[2][64], l[2][64];
    int last;
};

}  // namespace

// Grid (tiles * kv_heads, splits), four waves.  A tile is 16 rows of one head of
// the cache: rows are the queries of one sequence times the heads that share
// the cache head, in that order (with LIST, those of one token).  The waves take
// the pages of their workgroup's split in turn, each with the whole 16 rows, and
// join their states at the end; the last split of a tile to finish joins all of
// them, in the order of the splits, so that results do not depend on timing.
//
// Keys are the first operand and queries the second, so that a lane's scores
// belong to one row and the weights leave the softmax as the second operand of
// the product with the values; no weight and no score crosses lanes.
template <typename E, int D, bool LIST>
__global__ __launch_bounds__(kThreads, 2) void attend16_kernel(AttendParams p) {
    __shared__ Shared<E, D> sh;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % p.kv_heads, slot = blockIdx.x / p.kv_heads, split = blockIdx.y;

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
        // a sequence's tiles begin at floor(rows before it / 16) + its index:
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
    const int row = base + row0 + n;
    const int i = row / p.group, hq = head * p.group + row % p.group;
    const bool mine = n < valid;
    const Span span = visible(seq, i, p.causal, p.window);
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

    Queries<E, D> q;
    load_queries<E, D>(q,
                       (const typename E::T *)p.q + (int64_t)(seq.start + i) * p.q_token +
                           (int64_t)hq * p.q_head,
                       mine, g);

    RowState<D> st;
    st.m = -1e30f;   // finite: a row that has seen nothing weighs exp2(-inf) = 0
    st.l = 0.0f;
#pragma unroll
    for (int m = 0; m < D / 16; ++m) st.o[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int32_t *named =
        LIST ? p.named + ((int64_t)(seq.start + base / p.group) * p.kv_heads + head) * p.list
             : nullptr;
    const int32_t *table = p.table + (int64_t)seq.index * p.width;
    const int64_t stride = (int64_t)p.kv_heads * Record<D>::kBytes;
    const uint8_t *cache = p.cache + (int64_t)head * Record<D>::kBytes;
    const int last_page = (z.hi + kPage - 1) / kPage;

    for (int from = begin + wave; from < end; from += kWaves * 64) {
        // 64 of this wave's pages at a time, one a lane
        const int e = from + kWaves * lane;
        int page = -1, phys = -1;
        if (e < end) {
            page = LIST ? named[e] : page0 + e;
            if (page >= 0 && page < last_page) phys = table[page];
        }
        uint64_t todo = __builtin_amdgcn_ballot_w64(phys >= 0 && phys < p.pages);
        if (!todo) continue;
        PageRegs<D> cur;
        int at = __builtin_ctzll(todo);
        todo &= todo - 1;
        int number = __builtin_amdgcn_readlane(page, at);
        load_page<D>(cur, cache + (int64_t)__builtin_amdgcn_readlane(phys, at) * stride, n, g);
        while (true) {
            PageRegs<D> next;
            int next_number = -1;
            if (todo) {
                at = __builtin_ctzll(todo);
                todo &= todo - 1;
                next_number = __builtin_amdgcn_readlane(page, at);
                load_page<D>(next, cache + (int64_t)__builtin_amdgcn_readlane(phys, at) * stride, n,
                             g);
            }
            const int t0 = number * kPage;
            if (t0 < z.lo || t0 + kPage > a.hi)
                attend_page<E, D, true>(st, cur, q, p.scale_log2, span.lo - t0, span.hi - t0, g);
            else
                attend_page<E, D, false>(st, cur, q, p.scale_log2, 0, kPage, g);
            if (next_number < 0) break;
            cur = next;
            number = next_number;
        }
    }
    st.l = across_rows(st.l, [](float x, float y) { return x + y; });

    // join the waves: 2 and 3 into 0 and 1, then 1 into 0
#pragma unroll
    for (int half = kWaves / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half) {
            sh.m[wave - half][lane] = st.m;
            sh.l[wave - half][lane] = st.l;
#pragma unroll
            for (int m = 0; m < D / 16; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) sh.o[wave - half][4 * m + j][lane] = st.o[m][j];
        }
        __syncthreads();
        if (wave < half) {
            f32x4 o[D / 16];
#pragma unroll
            for (int m = 0; m < D / 16; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[m][j] = sh.o[wave][4 * m + j][lane];
            join<D>(st, sh.m[wave][lane], sh.l[wave][lane], o);
        }
        __syncthreads();
    }

    const int unit = blockIdx.x;
    constexpr int kPart = kRows * (D + 2);   // floats of a split: m[16], l[16], o[16][D]
    if (splits == 1) {
        if (wave == 0 && mine) {
            const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;
            const int64_t at = (int64_t)(seq.start + i) * (p.kv_heads * p.group) + hq;
            typename E::T *out = (typename E::T *)p.out + at * D + D / 16 * 4 * g;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int m = 0; m < D / 16; m += 2)
                    *reinterpret_cast<uint32_t *>(out + D / 16 * j + m) =
                        pack_pair<E>(st.o[m][j] * inv, st.o[m + 1][j] * inv);
            if (p.lse && g == 0)
                p.lse[at] = st.l == 0.0f ? -__builtin_inff()
                                         : (st.m + __builtin_log2f(st.l)) * 0.69314718055994531f;
        }
        return;
    }

    // several splits: leave this one's state in the workspace; the last to get
    // here joins them
    float *part = p.part + ((int64_t)unit * gridDim.y) * kPart;
    if (wave == 0) {
        float *my = part + (int64_t)split * kPart;
        if (mine) {
            if (g == 0) {
                my[n] = st.m;
                my[kRows + n] = st.l;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int m = 0; m < D / 16; m += 4)
                    *reinterpret_cast<f32x4 *>(my + 2 * kRows + n * D + D / 16 * (4 * g + j) + m) =
                        f32x4{st.o[m][j], st.o[m + 1][j], st.o[m + 2][j], st.o[m + 3][j]};
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
        if (lane == 0)
            sh.last = __hip_atomic_fetch_add(p.tickets + unit, 1, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT) == splits - 1;
    }
    __syncthreads();
    if (!sh.last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    if (threadIdx.x == 0) p.tickets[unit] = 0;   // for the next call
    for (int x = threadIdx.x; x < valid * (D / 4); x += kThreads) {
        const int r = x / (D / 4), c = x % (D / 4) * 4;
        float top = -1e30f;
        for (int s = 0; s < splits; ++s) top = fmaxf(top, part[(int64_t)s * kPart + r]);
        float l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; ++s) {
            const float *from = part + (int64_t)s * kPart;
            const float f = __builtin_amdgcn_exp2f(from[r] - top);
            l += from[kRows + r] * f;
            o += *reinterpret_cast<const f32x4 *>(from + 2 * kRows + r * D + c) * f;
        }
        const int rr = base + row0 + r;
        const int64_t at = (int64_t)(seq.start + rr / p.group) * (p.kv_heads * p.group) +
                           head * p.group + rr % p.group;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        u32x2 w = {pack_pair<E>(o[0] * inv, o[1] * inv), pack_pair<E>(o[2] * inv, o[3] * inv)};
        *reinterpret_cast<u32x2 *>((typename E::T *)p.out + at * D + c) = w;
        if (p.lse && c == 0)
            p.lse[at] = l == 0.0f ? -__builtin_inff()
                                  : (top + __builtin_log2f(l)) * 0.69314718055994531f;
    }
}

namespace {

template <typename E, int D>
void launch_d(const AttendParams &p, dim3 grid, hipStream_t s) {
    if (p.named)
        hipLaunchKernelGGL((attend16_kernel<E, D, true>), grid, dim3(kThreads), 0, s, p);
    else
        hipLaunchKernelGGL((attend16_kernel<E, D, false>), grid, dim3(kThreads), 0, s, p);
}

template <typename E>
void launch_t(const AttendParams &p, int dim, dim3 grid, hipStream_t s) {
    if (dim == 64) launch_d<E, 64>(p, grid, s);
    else if (dim == 128) launch_d<E, 128>(p, grid, s);
    else launch_d<E, 256>(p, grid, s);
}

}  // namespace

void launch_attend16(const AttendParams &p, int type, int dim, dim3 grid, hipStream_t s) {
    if (type == LCE_FLOAT16) launch_t<F16>(p, dim, grid, s);
    else launch_t<Bf16>(p, dim, grid, s);
}

}  // namespace kv4
}  // namespace lce
