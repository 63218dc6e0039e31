// Writing the 4-bit key/value cache and reading it back.
#include "kv4_launch.hpp"

namespace lce {
namespace kv4 {
namespace {

// Eight channels as they come from memory, and what the group's scale needs of
// them: the absolute values' bits, which as whole numbers are in the order of
// the values, infinities and NaN last.
template <typename T>
struct Eight;

template <>
struct Eight<float> {
    u32x4 w[2];
    __device__ __forceinline__ void load(const float *p) {
        w[0] = reinterpret_cast<const u32x4 *>(p)[0];
        w[1] = reinterpret_cast<const u32x4 *>(p)[1];
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i / 4][i % 4] & 0x7FFFFFFFu);
        return m;
    }
    // biased exponent of a float32 with the same power of two, 255 if not finite
    static __device__ __forceinline__ int exponent(uint32_t top) { return (int)(top >> 23); }
    __device__ __forceinline__ float value(int i) const { return bits_as<float>(w[i / 4][i % 4]); }
    template <int I>
    __device__ __forceinline__ uint32_t pack(uint32_t old, float scale) const {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, value(2 * I), value(2 * I + 1), scale,
                                                        I);
    }
    __device__ __forceinline__ uint32_t signs() const {
        uint32_t b = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) b |= (value(i) < 0.0f ? 1u : 0u) << i;
        return b;
    }
};

// float16 and bfloat16 share everything but the width of the exponent.
template <typename T, typename T2>
struct EightHalf {
    u32x4 w;
    __device__ __forceinline__ void load(const T *p) { w = *reinterpret_cast<const u32x4 *>(p); }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
        return m;
    }
    __device__ __forceinline__ T2 pair(int i) const { return bits_as<T2>((uint32_t)w[i]); }
    __device__ __forceinline__ uint32_t signs() const {
        uint32_t b = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            b |= ((float)pair(i)[0] < 0.0f ? 1u : 0u) << (2 * i);
            b |= ((float)pair(i)[1] < 0.0f ? 2u : 0u) << (2 * i);
        }
        return b;
    }
};

template <>
struct Eight<__bf16> : EightHalf<__bf16, bf16x2> {
    static __device__ __forceinline__ int exponent(uint32_t top) { return (int)(top >> 7); }
    template <int I>
    __device__ __forceinline__ uint32_t pack(uint32_t old, float scale) const {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, pair(I), scale, I);
    }
};

template <>
struct Eight<_Float16> : EightHalf<_Float16, f16x2> {
    static __device__ __forceinline__ int exponent(uint32_t top) {
        if (top >= 0x7C00u) return 255;
        // exact in float32, subnormal ones too
        return (int)(bits_as<uint32_t>((float)bits_as<_Float16>((uint16_t)top)) >> 23);
    }
    template <int I>
    __device__ __forceinline__ uint32_t pack(uint32_t old, float scale) const {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, pair(I), scale, I);
    }
};

template <typename E>
__device__ __forceinline__ uint32_t codes(const E &x, float scale) {
    uint32_t c = 0;
    c = x.template pack<0>(c, scale);
    c = x.template pack<1>(c, scale);
    c = x.template pack<2>(c, scale);
    return x.template pack<3>(c, scale);
}

// The largest over a group's four lanes (a quad): DPP quad permutes.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
}

// Byte offset in a record of the value codes of channels 8l .. 8l+7 of token t:
// 4 bytes, of which a head of 64 channels holds two pieces of 2.
template <int D>
__device__ __forceinline__ int value_offset(int t, int l) {
    constexpr int G = D / 32;   // bytes of a token under one r
    const int r = 8 * l / (D / 16), w = 8 * l % (D / 16);
    return Record<D>::kValue + ((t / 4 * 16 + r) * 4 + t % 4) * G + w / 2;
}

}  // namespace

// One thread per eight channels of a token's key and value, D/8 threads per
// token; a workgroup covers consecutive tokens of one head, so that the value
// codes, which interleave four tokens, and the scales, which interleave 64,
// leave a CU as whole lines.  U tokens per thread keep U*2 loads in flight.
// Bound by memory: reads 2*D elements, writes 19/16*D bytes a token and head.
// Measured: 12001 tokens, 8 heads of 128, float16 (64 MB) 14.0 us, 4.6 TB/s (a large
// copy: 5.35); 32 tokens 2.6 us, a launch.
template <typename T, int D, int U>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendParams p) {
    constexpr int L = D / 8, N = kThreads / L;
    const int l = threadIdx.x % L, head = blockIdx.x % p.kv_heads;
    const int64_t first = (int64_t)(blockIdx.x / p.kv_heads) * (N * U) + threadIdx.x / L;
    Eight<T> k[U], v[U];
    int64_t slot[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = min(first + u * N, p.tokens - 1);
        slot[u] = first + u * N < p.tokens ? p.slots[i] : -1;
        k[u].load((const T *)p.k + i * p.k_token + head * p.k_head + 8 * l);
        v[u].load((const T *)p.v + i * p.v_token + head * p.v_head + 8 * l);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int ke = Eight<T>::exponent(quad_max(k[u].top()));
        const int ve = Eight<T>::exponent(quad_max(v[u].top()));
        // lanes of this token whose groups are not finite
        const uint64_t odd = __builtin_amdgcn_ballot_w64(ke == 255 || ve == 255);
        const uint64_t mine = (L == 64 ? ~0ull : (1ull << (L & 63)) - 1)
                              << ((threadIdx.x & 63) / L * L);
        const bool whole = (odd & mine) == 0;
        const uint32_t kb = whole ? max(ke - 2, 0) : 255, vb = ve == 255 ? 255 : max(ve - 2, 0);
        const uint32_t kc = whole ? codes(k[u], scale_of(kb)) : 0;
        const uint32_t vc = ve == 255 ? 0 : codes(v[u], scale_of(vb));
        if (slot[u] < 0 || slot[u] >= (int64_t)p.pages * kPage) continue;
        uint8_t *rec = p.cache + ((slot[u] / kPage) * p.kv_heads + head) * (int64_t)Record<D>::kBytes;
        const int t = (int)(slot[u] % kPage);
        *reinterpret_cast<uint32_t *>(rec + Record<D>::kKey + t * (D / 2) + 4 * l) = kc;
        if constexpr (D == 64) {
            *reinterpret_cast<uint16_t *>(rec + value_offset<D>(t, l)) = (uint16_t)vc;
            *reinterpret_cast<uint16_t *>(rec + value_offset<D>(t, l) + 8) = (uint16_t)(vc >> 16);
        } else {
            *reinterpret_cast<uint32_t *>(rec + value_offset<D>(t, l)) = vc;
        }
        rec[Record<D>::kSigns + t * (D / 8) + l] = (uint8_t)k[u].signs();
        if (l % 4 == 0) {
            const int g = l / 4;
            rec[Record<D>::kKeyScale + (t % 16 * (D / 32) + g) * 4 + t / 16] = (uint8_t)kb;
            rec[Record<D>::kValueScale + g * 64 + t % 16 / 4 * 16 + t / 16 * 4 + t % 4] =
                (uint8_t)vb;
        }
    }
}

namespace {

// Eight values stored; LONG: past the caches.
template <bool LONG, typename V>
__device__ __forceinline__ void store16(void *p, const V &v) {
    if constexpr (LONG)
        __builtin_nontemporal_store(v, static_cast<V *>(p));
    else
        *static_cast<V *>(p) = v;
}

// Stores the eight values of each of the L lanes of a token at `p`, the token's
// first channel; every lane of the wave takes part.  Two bytes a value: a lane's
// eight are 16 bytes.  Four: a lane stores four values of the token's first half
// and four of its second, whose codes other lanes hold, so that a store of the
// wave is whole lines here too.
template <typename T, int L, bool LONG>
__device__ __forceinline__ void store_values(T *p, int l, uint32_t c, uint32_t scale, bool valid) {
    if constexpr (__is_same(T, float)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int from = (threadIdx.x & 63) / L * L + (l + j * L) / 2;
            const uint32_t w = (uint32_t)__shfl((int)c, from) >> (l % 2 * 16);
            const float s = scale_of((uint32_t)__shfl((int)scale, from));
            const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0);
            const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
            if (valid) store16<LONG>(p + 4 * (l + j * L), f32x4{x[0], x[1], y[0], y[1]});
        }
    } else {
        const float s = scale_of(scale);
        u32x4 w;
        if constexpr (__is_same(T, __bf16))
            w = u32x4{bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0)),
                      bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1)),
                      bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2)),
                      bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3))};
        else
            w = u32x4{bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 0)),
                      bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 1)),
                      bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 2)),
                      bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 3))};
        if (valid) store16<LONG>(p + 8 * l, w);
    }
}

}  // namespace

// The same split for reading: one thread per eight channels, 4 bytes of codes
// and one scale of each of key and value in, eight elements of each out.
// Bound by memory, mostly its writes.  Measured, 8 heads of 128: 65536 tokens to
// bfloat16 (340 MB) 50.8 us, 6.7 TB/s; 12001 tokens to float16 (62 MB) 11.6 us.
template <typename T, int D, int U, bool LONG>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadParams p) {
    constexpr int L = D / 8, N = kThreads / L;
    const int l = threadIdx.x % L, head = blockIdx.x % p.kv_heads, g = l / 4;
    const int64_t first = (int64_t)(blockIdx.x / p.kv_heads) * (N * U) + threadIdx.x / L;
    int64_t slot[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        slot[u] = first + u * N < p.tokens ? p.slots[first + u * N] : -1;
    uint32_t kc[U], vc[U], ks[U], vs[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        kc[u] = vc[u] = ks[u] = vs[u] = 0;   // outside the cache: 0 * 2^-127
        if (slot[u] < 0 || slot[u] >= (int64_t)p.pages * kPage) continue;
        const uint8_t *rec =
            p.cache + ((slot[u] / kPage) * p.kv_heads + head) * (int64_t)Record<D>::kBytes;
        const int t = (int)(slot[u] % kPage);
        kc[u] = *reinterpret_cast<const uint32_t *>(rec + Record<D>::kKey + t * (D / 2) + 4 * l);
        if constexpr (D == 64)
            vc[u] = *reinterpret_cast<const uint16_t *>(rec + value_offset<D>(t, l)) |
                    (uint32_t) * reinterpret_cast<const uint16_t *>(rec + value_offset<D>(t, l) + 8)
                        << 16;
        else
            vc[u] = *reinterpret_cast<const uint32_t *>(rec + value_offset<D>(t, l));
        ks[u] = rec[Record<D>::kKeyScale + (t % 16 * (D / 32) + g) * 4 + t / 16];
        vs[u] = rec[Record<D>::kValueScale + g * 64 + t % 16 / 4 * 16 + t / 16 * 4 + t % 4];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = first + u * N;
        const int64_t at = (i * p.kv_heads + head) * D;
        store_values<T, L, LONG>((T *)p.k + at, l, kc[u], ks[u], i < p.tokens);
        store_values<T, L, LONG>((T *)p.v + at, l, vc[u], vs[u], i < p.tokens);
    }
}

namespace {

// Four tokens a thread where that still gives every CU a few workgroups (the
// loads of the four are in flight together); one where the call is so short
// that the number of workgroups is what it lacks.
bool four_per_thread(int64_t tokens, int heads, int dim) {
    return tokens * heads * (dim / 8) >= (int64_t)1024 * kThreads * 4;
}

// Workgroups of u tokens a thread, of one head.
template <typename P>
dim3 grid_of(const P &p, int dim, int u) {
    const int64_t per = (int64_t)kThreads / (dim / 8) * u;
    return dim3((unsigned)((p.tokens + per - 1) / per * p.kv_heads));
}

template <typename T, int D>
void launch_append_d(const AppendParams &p, hipStream_t s) {
    if (four_per_thread(p.tokens, p.kv_heads, D))
        hipLaunchKernelGGL((append_kernel<T, D, 4>), grid_of(p, D, 4), dim3(kThreads), 0, s, p);
    else
        hipLaunchKernelGGL((append_kernel<T, D, 1>), grid_of(p, D, 1), dim3(kThreads), 0, s, p);
}

// Results of more than 100 MB are stored past the caches, which would not hold them
// for whoever reads them next.  Measured, bfloat16, 8 heads of 128 (us, with and
// without; then with a pass over the keys behind it): 98 MB 20.4, 19.9 (36.7,
// 37.5), 134 MB 31.2, 26.2 (51.4, 49.3), 268 MB 76.3, 50.4.
template <typename T, int D>
void launch_read_d(const ReadParams &p, hipStream_t s) {
    const int64_t bytes = p.tokens * p.kv_heads * 2 * D * (int64_t)sizeof(T);
    if (bytes > 100 << 20)
        hipLaunchKernelGGL((read_kernel<T, D, 4, true>), grid_of(p, D, 4), dim3(kThreads), 0, s, p);
    else if (four_per_thread(p.tokens, p.kv_heads, D))
        hipLaunchKernelGGL((read_kernel<T, D, 4, false>), grid_of(p, D, 4), dim3(kThreads), 0, s, p);
    else
        hipLaunchKernelGGL((read_kernel<T, D, 1, false>), grid_of(p, D, 1), dim3(kThreads), 0, s, p);
}

template <typename T>
void launch_append_t(const AppendParams &p, int dim, hipStream_t s) {
    if (dim == 64) launch_append_d<T, 64>(p, s);
    else if (dim == 128) launch_append_d<T, 128>(p, s);
    else launch_append_d<T, 256>(p, s);
}

template <typename T>
void launch_read_t(const ReadParams &p, int dim, hipStream_t s) {
    if (dim == 64) launch_read_d<T, 64>(p, s);
    else if (dim == 128) launch_read_d<T, 128>(p, s);
    else launch_read_d<T, 256>(p, s);
}

}  // namespace

void launch_append(const AppendParams &p, int type, int dim, hipStream_t s) {
    if (type == LCE_FLOAT32) launch_append_t<float>(p, dim, s);
    else if (type == LCE_FLOAT16) launch_append_t<_Float16>(p, dim, s);
    else launch_append_t<__bf16>(p, dim, s);
}

void launch_read(const ReadParams &p, int type, int dim, hipStream_t s) {
    if (type == LCE_FLOAT32) launch_read_t<float>(p, dim, s);
    else if (type == LCE_FLOAT16) launch_read_t<_Float16>(p, dim, s);
    else launch_read_t<__bf16>(p, dim, s);
}

}  // namespace kv4
}  // namespace lce
