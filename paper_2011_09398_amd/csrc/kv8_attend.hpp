// What the attention kernels over the 8-bit cache share.
#pragma once

#include "kv8.hpp"

namespace lce {
namespace kv8 {

// Codes are multiplied in the queries' type, times a power of two that brings the largest
// scale of what is multiplied together to 2^kUp: bfloat16 then holds every code of every
// scale that counts, float16 every code whose scale is down to 2^-22 of the largest, and
// smaller ones to 2^-25 (of 448 * 2^7).
template <typename E>
constexpr int kUp = __is_same(E, F16) ? 7 : 0;

// Two codes (the low or the high half of w) as a packed pair of E::T, times s, a power of two.
template <typename E, bool HIGH>
__device__ __forceinline__ uint32_t decode_codes(uint32_t w, float s) {
    if constexpr (__is_same(E, F16))
        return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, HIGH));
    else
        return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, HIGH));
}

template <typename E>
__device__ __forceinline__ u32x4 decode_eight(uint32_t a, uint32_t b, float sa, float sb) {
    return u32x4{decode_codes<E, false>(a, sa), decode_codes<E, true>(a, sa),
                 decode_codes<E, false>(b, sb), decode_codes<E, true>(b, sb)};
}

// 2^(e - of + up) for scale bytes e <= of (2^-126 where it would be less).
__device__ __forceinline__ float relative(int e, int of, int up) {
    return bits_as<float>((uint32_t)max(127 + e - of + up, 1) << 23);
}

// What the scores of keys whose largest scale byte is `most` are multiplied by: finite, so
// that a score of 0 stays one, and more than 0, so that a hidden token's of -infinity does.
// (2^-149 at least, which is within 2^-21 of what any finite score times less would be.
// Positive floats are in the order of their bits.)
template <typename E>
__device__ __forceinline__ float score_factor(float scale_log2, int most) {
    const float f = __builtin_amdgcn_ldexpf(scale_log2, most - 127 - kUp<E>);
    return bits_as<float>(max(bits_as<uint32_t>(__builtin_fminf(f, __FLT_MAX__)), 1u));
}

// Two query channels of type E::T, infinities as NaNs: an infinity times a key is one or the
// other infinity, which as a score may be below all (and weigh nothing) or be capped, a NaN
// makes its row one whatever it is multiplied by.
template <typename E>
__device__ __forceinline__ uint32_t without_infinities(uint32_t w) {
    if constexpr (__is_same(E, F16)) {
        const f16x2 x = bits_as<f16x2>(w);
        return bits_as<uint32_t>(__builtin_elementwise_fma(x, f16x2{0, 0}, x));
    } else {
        // exponents of all ones carry into the sign's place, from there to the quiet bit
        return w | ((((w & 0x7F807F80u) + 0x00800080u) >> 9) & 0x00400040u);
    }
}

// The scale bytes (byte i: block i) of a page of which some row sees tokens [lo, hi):
// blocks that no row sees weigh next to nothing, whatever their bytes are.
__device__ __forceinline__ uint32_t settled_scales(uint32_t scales, int lo, int hi) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
        const bool seen = kBlock * i < hi && kBlock * (i + 1) > lo;
        const uint32_t e = (uint32_t)clampi((int)(scales >> (8 * i) & 255u), kLeastScale, kMostScale);
        w |= (seen ? e : (uint32_t)kLeastScale) << (8 * i);
    }
    return w;
}

// A value that all lanes have, in a scalar register (or what is made of it would be made in
// all lanes).
__device__ __forceinline__ uint32_t in_scalar(uint32_t x) {
    uint32_t s = (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
    asm volatile("" : "+s"(s));
    return s;
}

__device__ __forceinline__ int byte_of(uint32_t w, int i) { return (int)(w >> (8 * i) & 255u); }

__device__ __forceinline__ int largest_of(uint32_t w) {
    return max(max(byte_of(w, 0), byte_of(w, 1)), max(byte_of(w, 2), byte_of(w, 3)));
}

// The bytes of a word of value codes, tokens first .. first + 3, that some row sees, [lo,
// hi) being what some row sees: the others may be anything, and a weight of 0 times a NaN
// is not 0.
__device__ __forceinline__ uint32_t seen_bytes(int first, int lo, int hi) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (first + i >= lo && first + i < hi) w |= 255u << (8 * i);
    return w;
}

// A sum, and two weights in the type in which they multiply values.
__device__ __forceinline__ float add_rounded(Bf16, uint32_t w, float sum) {
    constexpr bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(bits_as<bf16x2>(w), one, sum, false);
}

__device__ __forceinline__ float add_rounded(F16, uint32_t w, float sum) {
    constexpr f16x2 one = {(_Float16)1.0f, (_Float16)1.0f};
    return __builtin_amdgcn_fdot2(bits_as<f16x2>(w), one, sum, false);
}

// What a call does to scores between their product and the softmax: nothing, a cap of up to
// kNearCap, a bias by distance, or another cap or both.  (The first three have kernels of their
// own because values that several branches make are copied where these meet: the prompts of
// the 16-row kernel's comment 52 us in the last's, 47 in their own.)
enum class Change { kNone, kCapped, kSloped, kAny };
constexpr bool has_slopes(Change c) { return c == Change::kSloped || c == Change::kAny; }
constexpr float kNearCap = 256.0f;         // log2 units
static_assert(kNearCap + kLag + F16::kLift < kLarge, "capped scores are not large");

struct Cap {
    float cap, inverse;    // log2 units, 0: none; 1 / cap

    // Caps scores, which times `by` are in log2 units: each(f) puts f(x) in the place of
    // every score x, and what times `by` plus `offset` is in log2 units is then
    // cap * tanh(u), as cap (1 - 2 / (exp(2u) + 1)), whose ends, exponentials of 0 and
    // infinity, give -1 and 1, known to 2^-22 of the cap.  That is enough of caps in use; under
    // large ones small u take the power series (|u| < 1/4: up to u^9, off by less than 2^-26
    // of it).
    template <Change C, typename Each>
    __device__ __forceinline__ void limit(float &by, float &offset, Each each) const {
        // (finite: a score of 0 stays one)
        const float u1 = by * inverse;
        const float twice = __builtin_fminf(u1 * 2.88539008177792681f, __FLT_MAX__);
        const auto part = [&](float x) {
            return __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(x * twice));
        };
        if constexpr (C == Change::kCapped) {
            each(part);
            by = 2.0f * cap;
            offset = cap;
            return;
        }
        const auto far = [&](float x) { return __builtin_fmaf(2.0f * cap, part(x), cap); };
        if (cap <= kNearCap) {
            each(far);
        } else {
            each([&](float x) {
                const float y = x * by, u = x * u1, z = u * u;
                float t = __builtin_fmaf(z, 62.0f / 2835, -17.0f / 315);
                t = __builtin_fmaf(z, t, 2.0f / 15);
                t = __builtin_fmaf(z, t, -1.0f / 3);
                t = __builtin_fmaf(z * t, y, y);
                return z < 0.0625f ? t : far(x);
            });
        }
        by = 1.0f;
    }
};

// A lane's row, for a bias by distance.
struct Slope {
    float slope;           // log2 units a token
    int position;

    __device__ __forceinline__ void set(float nats, int at) {
        slope = nats * 1.44269504088896341f;
        position = at;
    }
    // (Of positions past 2^24 the distance is off by a last place, as it would be rounded to
    // float32 itself.)
    __device__ __forceinline__ float from(int token) const { return (float)(position - token); }
    __device__ __forceinline__ float operator()(float x, float distance) const {
        return __builtin_fmaf(-slope, __builtin_fabsf(distance), x);
    }
};

// A split's state in the workspace: of each row its maximum and its sum of weights, the scale
// byte of its sums of values and what they are divided by, then the sums of four channels at a
// time, `rows` rows next to each other.
template <int D, int ROWS>
struct Part {
    static constexpr int kFloats = ROWS * (D + 4);
    static __device__ __forceinline__ int state(int row) { return 4 * row; }
    static __device__ __forceinline__ int sums(int rows, int row, int quad) {
        return 4 * ROWS + 4 * (quad * rows + row);
    }
};

// Four channels of a row over all its splits, sixteen splits at a time, each with its own
// maximum and scale, against running ones.
struct Joined {
    f32x4 o;
    float top, l, divisor;
    int scale;
};

template <int D, int ROWS>
__device__ __forceinline__ Joined join_parts(const float *part, int splits, int rows, int row,
                                             int quad) {
    typedef Part<D, ROWS> P;
    Joined r;
    r.o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    r.top = kNone;
    r.l = r.divisor = 0.0f;
    r.scale = kLeastScale;
    for (int s0 = 0; s0 < splits; s0 += 16) {
        f32x2 ml[16];
        f32x2 divisor[16];                     // and the scale byte before it
        f32x4 y[16];
        // four at a time are there or not: what is past the last split is read again,
        // and weighs nothing
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            ml[k] = f32x2{kNone, 0.0f};
            divisor[k] = f32x2{(float)kLeastScale, 0.0f};
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
                    divisor[k] = got(from + P::state(row) + 2);
                    y[k] = f32x4{a[0], a[1], b[0], b[1]};
                }
            }
        float high = r.top;
        int most = r.scale;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            high = fmaxf(high, ml[k][0]);
            most = max(most, (int)divisor[k][0]);
        }
        const float f = __builtin_amdgcn_exp2f(r.top - high);
        r.l *= f;
        r.divisor *= f;
        r.o *= f * relative(r.scale, most, 0);
        r.top = high;
        r.scale = most;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float w = s0 + k < splits ? __builtin_amdgcn_exp2f(ml[k][0] - r.top) : 0.0f;
            r.l += ml[k][1] * w;
            r.divisor += divisor[k][1] * w;
            r.o += y[k] * (w * relative((int)divisor[k][0], most, 0));
        }
    }
    return r;
}

// Four channels of a row's result, and the log of its sum.
template <typename E>
__device__ __forceinline__ u32x2 result(const f32x4 &o, float divisor, int scale) {
    const float inv = divisor == 0.0f ? 0.0f : 1.0f / divisor;
    // codes' means are at most 448 * 2^kUp: only the last factor leaves float32's middle
    const int e = scale - 127 - kUp<E>;
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_ldexpf(o[i] * inv, e);
    return u32x2{pack_result<E>(x[0], x[1]), pack_result<E>(x[2], x[3])};
}

__device__ __forceinline__ float log_sum(float top, float l) {
    return l == 0.0f ? -__builtin_inff() : (top + __builtin_log2f(l)) * 0.69314718055994531f;
}

// The kernel that a call takes, by what it does to scores: launch(kind), kind::value being
// a Change.
template <Change C>
struct ChangeOf {
    static constexpr Change value = C;
};

template <typename Launch>
void by_change(const AttendParams &p, Launch launch) {
    if (p.slopes && p.cap_log2 == 0.0f) launch(ChangeOf<Change::kSloped>());
    else if (p.slopes || p.cap_log2 > kNearCap) launch(ChangeOf<Change::kAny>());
    else if (p.cap_log2 > 0.0f) launch(ChangeOf<Change::kCapped>());
    else launch(ChangeOf<Change::kNone>());
}

}  // namespace kv8
}  // namespace lce
