// Writing the 8-bit key/value cache and reading it back.
#include "kv8.hpp"

namespace lce {
namespace kv8 {
namespace {

constexpr int kWaves = kThreads / 64;

// N consecutive channels as they come from memory: 16 bytes at a time, or 8.
template <typename T, int N>
struct Channels {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];

    __device__ __forceinline__ void load(const T *p) {
        if constexpr (kWords == 2) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
            w[0] = x[0], w[1] = x[1];
        } else {
#pragma unroll
            for (int j = 0; j < kWords / 4; ++j) {
                const u32x4 x = reinterpret_cast<const u32x4 *>(p)[j];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[4 * j + i] = x[i];
            }
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    // the value of channel i as the bits of a float32
    __device__ __forceinline__ uint32_t bits(int i) const {
        if constexpr (sizeof(T) == 4) return w[i];
        else if constexpr (__is_same(T, __bf16)) return i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16;
        else return bits_as<uint32_t>((float)bits_as<f16x2>(w[i / 2])[i % 2]);
    }
};

// The largest over the wave's 64 lanes, in all of them.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, true));   // row_ror:1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, true));
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

// The smallest scale with which the value of these bits is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(uint32_t top) {
    return clampi((int)((top + 0x1FFFFFu) >> 23) - 8, kLeastScale, kMostScale);
}

// 2^-(byte - 127), exact for scales in range.
__device__ __forceinline__ float inverse_scale(int byte) {
    return bits_as<float>((uint32_t)(254 - byte) << 23);
}

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

constexpr uint32_t kNan4 = 0x7F7F7F7Fu;   // key codes of a token that holds no number

// Four codes times a power of two that is at most 1.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return pack4(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t *p) {
    if constexpr (N == 1) w[0] = *reinterpret_cast<const uint32_t *>(p);
    else if constexpr (N == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
        w[0] = x[0], w[1] = x[1];
    } else {
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            const u32x4 x = reinterpret_cast<const u32x4 *>(p)[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[4 * j + i] = x[i];
        }
    }
}

template <int N>
__device__ __forceinline__ void store_words(uint8_t *p, const uint32_t (&w)[N]) {
    if constexpr (N == 1) *reinterpret_cast<uint32_t *>(p) = w[0];
    else if constexpr (N == 2) *reinterpret_cast<u32x2 *>(p) = u32x2{w[0], w[1]};
    else {
#pragma unroll
        for (int j = 0; j < N / 4; ++j)
            reinterpret_cast<u32x4 *>(p)[j] = u32x4{w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]};
    }
}

}  // namespace

// One wave per block of 16 tokens and head.  Lane (n, g), n = lane % 16, g = lane / 16,
// has D/16 channels from D/16 * n on of the block's tokens 4g .. 4g + 3: of the values,
// whole words of four tokens.  The new tokens' largest absolute value gives the scale, or
// the scale that the block's older tokens have, where that is larger; where it is smaller,
// their codes are rounded again.
// Bound by memory: reads 2*D elements a token and head, writes 2*D bytes.  Measured, 8
// heads of 128: 10900 new tokens of 7 sequences, float16 (67 MB) 16 us, of which the loads
// in a row (lengths, table, tokens) take 4; one token of each of 32 sequences 5 us.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendParams p) {
    constexpr int N = D / 16, W = N / 4;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int64_t item =
        (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const int head = (int)(item % p.kv_heads);
    const int64_t unit = item / p.kv_heads;
    // a sequence's blocks begin at floor(tokens before it / 16) + 2 * its index: its n new
    // tokens touch at most floor(n / 16) + 2 of them, and none is shared
    const auto first = [](int s, int b) { return (int64_t)s / kBlock + 2 * (int64_t)b; };
    const Sequence s = find_sequence(p.q_start, p.lengths, p.seqs, p.tokens, p.width, unit, first);
    if (s.index < 0) return;
    const int p0 = s.length - s.queries;                 // of the first new token; may be < 0
    const int64_t wide = max(p0, 0) / kBlock + (unit - first(s.start, s.index));
    if (wide * kBlock >= s.length) return;
    const int b0 = (int)wide * kBlock;                   // the block's first position
    const int held = clampi(p0 - b0, 0, kBlock);         // its older tokens
    const int end = min(s.length - b0, kBlock);
    const int phys = p.table[(int64_t)s.index * p.width + b0 / kPage];

    Channels<T, N> k[4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = 4 * g + i;
        k[i].clear(), v[i].clear();
        if (t >= held && t < end) {
            const int64_t token = s.start + (b0 + t - p0);
            k[i].load((const T *)p.k + token * p.k_token + head * p.k_head + N * n);
            v[i].load((const T *)p.v + token * p.v_token + head * p.v_head + N * n);
        }
    }
    if (phys < 0 || phys >= p.pages) return;
    uint8_t *rec = p.cache + ((int64_t)phys * p.kv_heads + head) * Record<D>::kBytes;
    const int block = b0 % kPage / kBlock;
    uint8_t *keys = rec + Record<D>::kKey + (kBlock * block + 4 * g) * D + N * n;
    uint8_t *values = rec + Record<D>::kValue + (4 * block + g) * 4 * D + 4 * N * n;
    uint8_t *scales = rec + Record<D>::kScale + block;

    // tokens that hold an infinity or a NaN, in any lane of a row
    uint32_t ktop = 0, vtop = 0;
    bool odd[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t mine = 0, bad = 0, most = 0;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const uint32_t x = k[i].bits(c) & 0x7FFFFFFFu, y = v[i].bits(c) & 0x7FFFFFFFu;
            mine = max(mine, x);
            bad = max(bad, max(x, y));
            most = max(most, y < 0x7F800000u ? y : 0u);
        }
        const uint64_t any = __builtin_amdgcn_ballot_w64(bad >= 0x7F800000u);
        odd[i] = (any >> (16 * g) & 0xFFFFu) != 0;
        ktop = max(ktop, odd[i] ? 0u : mine);
        vtop = max(vtop, most);
    }
    int kb = scale_byte(wave_max(ktop)), vb = scale_byte(wave_max(vtop));
    float kagain = 1.0f, vagain = 1.0f;                  // what older codes are multiplied by
    bool kgrew = false, vgrew = false;
    if (held) {
        const int kwas = clampi(scales[0], kLeastScale, kMostScale);
        const int vwas = clampi(scales[kBlocks], kLeastScale, kMostScale);
        kgrew = kb > kwas, vgrew = vb > vwas;
        kb = max(kb, kwas), vb = max(vb, vwas);
        // (at least 2^-126: beyond that nothing is left of any code)
        kagain = bits_as<float>((uint32_t)max(127 + kwas - kb, 1) << 23);
        vagain = bits_as<float>((uint32_t)max(127 + vwas - vb, 1) << 23);
    }
    const float kinv = inverse_scale(kb), vinv = inverse_scale(vb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = 4 * g + i;
        uint32_t w[W];
        if (t >= held && t < end) {
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const auto x = [&](int c) { return bits_as<float>(k[i].bits(4 * j + c)) * kinv; };
                w[j] = odd[i] ? kNan4 : pack4(x(0), x(1), x(2), x(3));
            }
            store_words<W>(keys + i * D, w);
        } else if (t < held && kgrew) {
            load_words<W>(w, keys + i * D);
#pragma unroll
            for (int j = 0; j < W; ++j) w[j] = w[j] == kNan4 ? kNan4 : rescale4(w[j], kagain);
            store_words<W>(keys + i * D, w);
        }
    }
    if (4 * g < end && (vgrew || 4 * g + 4 > held)) {
        uint32_t w[N];
#pragma unroll
        for (int c = 0; c < N; ++c) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t y = v[i].bits(c);
                x[i] = (y & 0x7FFFFFFFu) < 0x7F800000u ? bits_as<float>(y) * vinv : 0.0f;
            }
            w[c] = pack4(x[0], x[1], x[2], x[3]);
        }
        if (4 * g < held) {
            const int old = min(held - 4 * g, 4);        // older tokens of the word
            const uint32_t mask = old == 4 ? ~0u : (1u << (8 * old)) - 1;
            uint32_t was[N];
            load_words<N>(was, values);
#pragma unroll
            for (int c = 0; c < N; ++c)
                w[c] = ((vgrew ? rescale4(was[c], vagain) : was[c]) & mask) | (w[c] & ~mask);
        }
        store_words<N>(values, w);
    }
    if (lane == 0) {
        scales[0] = (uint8_t)kb;
        scales[kBlocks] = (uint8_t)vb;
    }
}

namespace {

// Eight values of a type; LONG: stored past the caches.
template <typename T, bool LONG>
__device__ __forceinline__ void store8(T *p, const float (&x)[8]) {
    u32x4 w[sizeof(T) / 2];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i / 4][i % 4] = bits_as<uint32_t>(x[i]);
    } else if constexpr (__is_same(T, __bf16)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[0][i] = pack_pair<Bf16>(x[2 * i], x[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[0][i] = pack_pair<F16>(x[2 * i], x[2 * i + 1]);
    }
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) {
        if constexpr (LONG) __builtin_nontemporal_store(w[j], reinterpret_cast<u32x4 *>(p) + j);
        else reinterpret_cast<u32x4 *>(p)[j] = w[j];
    }
}

__device__ __forceinline__ void unpack8(float (&x)[8], uint32_t lo, uint32_t hi, float s) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int w = (int)(j ? hi : lo);
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
        const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        x[4 * j] = a[0] * s, x[4 * j + 1] = a[1] * s, x[4 * j + 2] = b[0] * s, x[4 * j + 3] = b[1] * s;
    }
}

}  // namespace

// One thread per eight channels of a token; U tokens a thread.  Of the values, which
// interleave four tokens, it reads the words of all four and takes a byte of each: the
// tokens beside it find them in the cache.  Bound by memory, mostly its writes.  Measured, 8
// heads of 128: 40000 tokens to bfloat16 (246 MB) 37 us, 6.7 TB/s; 10900 to float16 12 us.
template <typename T, int D, int U, bool LONG>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadParams p) {
    constexpr int L = D / 8, N = kThreads / L;
    const int l = threadIdx.x % L, head = blockIdx.x % p.kv_heads;
    const int64_t first = (int64_t)(blockIdx.x / p.kv_heads) * (N * U) + threadIdx.x / L;
    int64_t slot[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        slot[u] = first + u * N < p.tokens ? p.slots[first + u * N] : -1;
    u32x2 k[U];
    u32x4 v[U][2];
    uint32_t ks[U], vs[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        k[u] = u32x2{0, 0};                       // outside the cache: 0 * 2^0
        v[u][0] = v[u][1] = u32x4{0, 0, 0, 0};
        ks[u] = vs[u] = 127;
        if (slot[u] < 0 || slot[u] >= (int64_t)p.pages * kPage) continue;
        const uint8_t *rec =
            p.cache + ((slot[u] / kPage) * p.kv_heads + head) * (int64_t)Record<D>::kBytes;
        const int t = (int)(slot[u] % kPage);
        k[u] = *reinterpret_cast<const u32x2 *>(rec + Record<D>::kKey + t * D + 8 * l);
        const u32x4 *at =
            reinterpret_cast<const u32x4 *>(rec + Record<D>::kValue + (t / 4 * D + 8 * l) * 4);
        v[u][0] = at[0], v[u][1] = at[1];
        ks[u] = rec[Record<D>::kScale + t / kBlock];
        vs[u] = rec[Record<D>::kScale + kBlocks + t / kBlock];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = first + u * N;
        if (i >= p.tokens) continue;
        const int64_t at = (i * p.kv_heads + head) * D + 8 * l;
        // byte t % 4 of each word
        const uint32_t b = (uint32_t)slot[u] % 4, pick = 0x0C0C0400u + b * 0x0101u;
        const auto four = [&](const u32x4 &w) {
            return __builtin_amdgcn_perm(w[1], w[0], pick) |
                   __builtin_amdgcn_perm(w[3], w[2], pick) << 16;
        };
        float x[8];
        unpack8(x, k[u][0], k[u][1], scale_of(ks[u]));
        store8<T, LONG>((T *)p.k + at, x);
        unpack8(x, four(v[u][0]), four(v[u][1]), scale_of(vs[u]));
        store8<T, LONG>((T *)p.v + at, x);
    }
}

namespace {

// Four tokens a thread where that still gives every CU a few workgroups (the loads of the
// four are in flight together).
bool four_per_thread(int64_t tokens, int heads, int dim) {
    return tokens * heads * (dim / 8) >= (int64_t)1024 * kThreads * 4;
}

template <typename T, int D>
void launch_append_d(const AppendParams &p, hipStream_t s) {
    hipLaunchKernelGGL((append_kernel<T, D>), dim3((unsigned)((p.items + kWaves - 1) / kWaves)),
                       dim3(kThreads), 0, s, p);
}

template <typename T, int D>
void launch_read_d(const ReadParams &p, hipStream_t s) {
    const auto grid = [&](int u) {
        const int64_t per = (int64_t)kThreads / (D / 8) * u;
        return dim3((unsigned)((p.tokens + per - 1) / per * p.kv_heads));
    };
    // results of more than 100 MB are stored past the caches, which would not hold them for
    // whoever reads them next (as measured for the 4-bit cache, whose results are the same)
    const int64_t bytes = p.tokens * p.kv_heads * 2 * D * (int64_t)sizeof(T);
    if (bytes > 100 << 20)
        hipLaunchKernelGGL((read_kernel<T, D, 4, true>), grid(4), dim3(kThreads), 0, s, p);
    else if (four_per_thread(p.tokens, p.kv_heads, D))
        hipLaunchKernelGGL((read_kernel<T, D, 4, false>), grid(4), dim3(kThreads), 0, s, p);
    else
        hipLaunchKernelGGL((read_kernel<T, D, 1, false>), grid(1), dim3(kThreads), 0, s, p);
}

template <typename T, typename P>
void launch_t(const P &p, int dim, hipStream_t s) {
    if constexpr (__is_same(P, AppendParams)) {
        if (dim == 64) launch_append_d<T, 64>(p, s);
        else if (dim == 128) launch_append_d<T, 128>(p, s);
        else launch_append_d<T, 256>(p, s);
    } else {
        if (dim == 64) launch_read_d<T, 64>(p, s);
        else if (dim == 128) launch_read_d<T, 128>(p, s);
        else launch_read_d<T, 256>(p, s);
    }
}

template <typename P>
void launch_any(const P &p, int type, int dim, hipStream_t s) {
    if (type == LCE_FLOAT32) launch_t<float>(p, dim, s);
    else if (type == LCE_FLOAT16) launch_t<_Float16>(p, dim, s);
    else launch_t<__bf16>(p, dim, s);
}

}  // namespace

void launch_append(const AppendParams &p, int type, int dim, hipStream_t s) {
    launch_any(p, type, dim, s);
}

void launch_read(const ReadParams &p, int type, int dim, hipStream_t s) {
    launch_any(p, type, dim, s);
}

}  // namespace kv8
}  // namespace lce
