// What the attention kernels over the 4-bit cache share: query operands,
// element types, and the joining of a row's splits.
#pragma once

#include "kv4_launch.hpp"

namespace lce {
namespace kv4 {

// Element type of queries, softmax weights and outputs, and its products.
struct Bf16 {
    typedef __bf16 T;
    typedef bf16x2 T2;
    typedef bf16x8 T8;
    // pieces of 4 significant bits (and a sign each) that hold any bfloat16
    static constexpr int kPieces = 2;
    static constexpr bool kSaturates = false;   // holds every finite cached value
    static constexpr float kLift = 0.0f;
    static __device__ __forceinline__ f32x4 mfma16(const u32x4 &a, const u32x4 &b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(bits_as<T8>(a), bits_as<T8>(b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(const u32x4 &a, const u32x4 &b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(bits_as<T8>(a), bits_as<T8>(b), c, 0, 0, 0);
    }
};

struct F16 {
    typedef _Float16 T;
    typedef f16x2 T2;
    typedef f16x8 T8;
    static constexpr int kPieces = 3;
    static constexpr bool kSaturates = true;    // cached values of 65536 and more: see below
    // Weights are taken against 2^-7 of the largest score's, so that they are at most
    // 2^15 (see kLag) and the small ones lose no bits above 2^-21 of the largest and
    // are not dropped above 2^-32, of which a long context has many.
    static constexpr float kLift = 7.0f;
    static __device__ __forceinline__ f32x4 mfma16(const u32x4 &a, const u32x4 &b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(bits_as<T8>(a), bits_as<T8>(b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(const u32x4 &a, const u32x4 &b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(bits_as<T8>(a), bits_as<T8>(b), c, 0, 0, 0);
    }
};

// Weights are taken against a maximum that follows the true one only when that has
// passed it by 2^kLag (beyond kLift): they cost no precision, and most pages then need
// neither the exchange between lanes nor the rescaling.
constexpr float kLag = 8.0f;

// The largest scale byte of a finite value: 6 * 2^125.
constexpr uint32_t kMaxScale = 252;

// Two codes (byte BYTE of c) as a packed pair of E::T, times a power of two; SAT: of
// float16's range, the nearest to it.
template <typename E, int BYTE, bool SAT = false>
__device__ __forceinline__ uint32_t decode_pair(uint32_t c, float s) {
    if constexpr (__is_same(typename E::T, __bf16)) {
        return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, BYTE));
    } else {
        f16x2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, BYTE);
        if constexpr (SAT) {
            constexpr f16x2 most = {(_Float16)65504.0f, (_Float16)65504.0f};
            x = __builtin_elementwise_max(__builtin_elementwise_min(x, most), -most);
        }
        return bits_as<uint32_t>(x);
    }
}

// What the scale bytes of the values of tokens first .. first + 3 (byte i: first + i)
// become on a page that not every row sees whole, [lo, hi) being what some row sees: a
// hidden token's weight is 0, and 0 times its values has to be 0.  Tokens that no row
// sees stand for next to nothing, whatever their bytes are, and those that some row
// sees for what they are; a group that is not finite has codes 0, and its key the NaN.
__device__ __forceinline__ uint32_t settled(uint32_t scale, int first, int lo, int hi) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (first + i >= lo && first + i < hi)
            w |= min(scale >> (8 * i) & 255u, kMaxScale) << (8 * i);
    return w;
}

// The highest bit of those of four scale bytes that are past 140, the largest with which
// every code is finite in float16: 6 * 2^13.  The values under such a scale are decoded
// with saturation (an infinity times a weight of 0 would be NaN), the others are spared
// its two instructions a pair.
__device__ __forceinline__ uint32_t past_float16(uint32_t scale) {
    return ((scale & 0x7F7F7F7Fu) + 0x73737373u) & scale & 0x80808080u;
}

// All bits of the bytes whose highest bit is set.
__device__ __forceinline__ uint32_t whole_bytes(uint32_t top) { return (top - (top >> 7)) | top; }

template <typename E>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
    typename E::T2 v = {(typename E::T)a, (typename E::T)b};
    return bits_as<uint32_t>(v);
}

// Two results.  They are means of values, which float16 holds; but their weights are
// rounded, and half a last place past 65504 is an infinity.  (NaN stays.)
template <typename E>
__device__ __forceinline__ uint32_t pack_result(float a, float b) {
    if constexpr (E::kSaturates) {
        const float most = 65504.0f;
        a = a > most ? most : a < -most ? -most : a;
        b = b > most ? most : b < -most ? -most : b;
    }
    return pack_pair<E>(a, b);
}

// A query is multiplied in 8-bit floats (e4m3) against the 4-bit keys, in groups of
// the same 32 channels that share a scale in a key.  With E = floor(log2 max|q|) of a
// group, the first piece is q * 2^(7-E) rounded to 4 significant bits, the next ones
// what is left, times 16 each: two hold a bfloat16's 8 bits exactly, three a float16's
// 11, of values down to 2^-13 of the group's largest, and smaller ones to 2^-21 and
// 2^-25 of it.  The matrix cores multiply the pieces' products by the pieces' scales and
// the key groups' own, so that products are exact but for that.
struct GroupScale {
    float up;         // 2^(7-E)
    uint32_t bytes;   // byte p: biased exponent of piece p, 2^(E-7-4p); 255 (NaN) for a
                      // group that is not finite
};

template <typename E>
__device__ __forceinline__ GroupScale group_scale(float top) {
    const uint32_t t = bits_as<uint32_t>(top);
    GroupScale r;
    // the smallest for which every piece's scale has an exponent; of bfloat16's groups
    // below it (2^-115), whose values are multiples of 2^-133, two pieces hold all bits
    constexpr int kLeast = 8 + 4 * (E::kPieces - 1);
    const int e = max((int)(t >> 23), kLeast);   // biased E
    r.up = bits_as<float>((uint32_t)(254 + 7 - e) << 23);
    r.bytes = 0;
#pragma unroll
    for (int p = 0; p < E::kPieces; ++p) r.bytes |= (uint32_t)(e - 7 - 4 * p) << (8 * p);
    if (t >= 0x7F800000u) r.bytes = ~0u;
    return r;
}

// The largest absolute value of those whose bits (without signs) `bits` is the largest
// of: bits are in the order of the values, infinities and NaN last.
template <typename E>
__device__ __forceinline__ float top_of(uint32_t bits) {
    const float top = (float)bits_as<typename E::T>((uint16_t)bits);
    return top < __builtin_inff() ? top : __builtin_inff();
}

// x of the lanes l and l^32: [0] is that of the one below 32.
__device__ __forceinline__ f32x2 both_halves(float x) {
    const auto a =
        __builtin_amdgcn_permlane32_swap(bits_as<uint32_t>(x), bits_as<uint32_t>(x), false, false);
    return f32x2{bits_as<float>((uint32_t)a[0]), bits_as<float>((uint32_t)a[1])};
}

// Four values -> four e4m3 bytes, and what the rounding left of them, times 16.
__device__ __forceinline__ uint32_t next_piece(float (&x)[4]) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[0] = (x[0] - lo[0]) * 16.0f;
    x[1] = (x[1] - lo[1]) * 16.0f;
    x[2] = (x[2] - hi[0]) * 16.0f;
    x[3] = (x[3] - hi[1]) * 16.0f;
    return (uint32_t)w;
}

// What workgroups on different XCDs tell each other within a launch is stored
// with relaxed atomics of device scope, which write through the caches that are
// not coherent; a release fence would write back the XCD's whole L2 instead, one
// workgroup after the other (64 ns each: 160 us of a launch of 2500, against 18).
// What remains of the order is that the stores are done before the ticket is
// drawn.  The one workgroup that reads them does so past the same caches, after a
// barrier behind the ticket: an acquire fence would empty them for all workgroups
// of the XCD, once for every unit (128 lists of 64 pages: 18.2 -> 16.6 us).
__device__ __forceinline__ void put(float *p, f32x2 v) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), bits_as<uint64_t>(v),
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ f32x2 got(const float *p) {
    return bits_as<f32x2>(__hip_atomic_load(reinterpret_cast<const uint64_t *>(p),
                                            __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Draws a ticket after this wave's stores; true for the last of `all`, which
// also puts the count back to 0 for the next call.
__device__ __forceinline__ bool last_of(int32_t *ticket, int all) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const int32_t before =
        __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before != all - 1) return false;
    __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

constexpr int kMostSplits = 256;   // of one unit

// A split's state in the workspace: (m, l) of each row, then sums four at a
// time in the order in which a wave holds them, `rows` rows next to each other,
// so that what a wave stores is one run of memory.
template <int D, int ROWS>
struct Part {
    static constexpr int kFloats = ROWS * (D + 4);
    static __device__ __forceinline__ int state(int row) { return 4 * row; }
    // sums `quad` (of D/4) of a row; which channels they are is the kernel's affair
    static __device__ __forceinline__ int sums(int rows, int row, int quad) {
        return 4 * ROWS + 4 * (quad * rows + row);
    }
};

// Joins sums `quad` of a row over all its splits, sixteen at a time, each with its
// own maximum, against a running one: the sums, their maximum and their weight.
template <int D, int ROWS>
__device__ __forceinline__ f32x4 join_splits(const float *part, int splits, int rows, int row,
                                             int quad, float &top, float &l) {
    typedef Part<D, ROWS> P;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    top = kNone;
    l = 0.0f;
    for (int s0 = 0; s0 < splits; s0 += 16) {
        f32x2 ml[16];
        f32x4 y[16];
        // four at a time are there or not: what is past the last split is read again,
        // and weighs nothing
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            ml[k] = f32x2{kNone, 0.0f};
            y[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
#pragma unroll
        for (int k0 = 0; k0 < 16; k0 += 4)
            if (s0 + k0 < splits) {
#pragma unroll
                for (int k = k0; k < k0 + 4; ++k) {
                    const float *from = part + (int64_t)min(s0 + k, splits - 1) * P::kFloats;
                    const float *sums = from + P::sums(rows, row, quad);
                    const f32x2 a = got(sums), b = got(sums + 2);
                    ml[k] = got(from + P::state(row));
                    y[k] = f32x4{a[0], a[1], b[0], b[1]};
                }
            }
        float high = top;
#pragma unroll
        for (int k = 0; k < 16; ++k) high = fmaxf(high, ml[k][0]);
        const float f = __builtin_amdgcn_exp2f(top - high);
        l *= f;
        o *= f;
        top = high;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float w = s0 + k < splits ? __builtin_amdgcn_exp2f(ml[k][0] - top) : 0.0f;
            l += ml[k][1] * w;
            o += y[k] * w;
        }
    }
    return o;
}

}  // namespace kv4
}  // namespace lce
