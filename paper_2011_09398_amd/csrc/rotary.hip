// Rotary positions: queries and keys turned by angles that grow with their tokens'
// positions.  C ABI (declared in lce.h), host-side checks and kernel.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdlib>

#include "status.hpp"

namespace {

using lce::aligned;
using lce::check_launch;
using lce::fail;
using lce::ok;

constexpr int kThreads = 256;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

// One tensor of a call: [tokens][heads][dim] from x to y, strides in elements.
struct Rows {
    const void *x;
    void *y;
    int64_t x_token, x_head, y_token, y_head;
    int heads;
};

struct RotaryParams {
    Rows rows[2];
    const uint64_t *turns;
    const int64_t *positions;
    int64_t items;
    int dim, rot, interleaved, backward;
    int lanes;        // lanes that share a token's heads
    int units;        // of a head, see Span
    int turned;       // units that are turned, before those that are copied
    float factor;
};

// N elements of T as they lie in memory (16 bytes of them, or one).
template <typename T, int N>
struct Span {
    u32x4 w;
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (N == 1)
            w[0] = __builtin_bit_cast(uint32_t, (float)*p);
        else
            w = *reinterpret_cast<const u32x4 *>(p);
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (N == 1)
            *p = (T)__builtin_bit_cast(float, (uint32_t)w[0]);
        else
            *reinterpret_cast<u32x4 *>(p) = w;
    }
    template <int I>
    __device__ __forceinline__ float get() const {
        if constexpr (sizeof(T) == 4 || N == 1)
            return __builtin_bit_cast(float, (uint32_t)w[I]);
        else if constexpr (__is_same(T, __bf16))
            return (float)__builtin_bit_cast(bf16x2, (uint32_t)w[I / 2])[I % 2];
        else
            return (float)__builtin_bit_cast(f16x2, (uint32_t)w[I / 2])[I % 2];
    }
    // elements I and I + 1 (N == 1 or four bytes each: I alone)
    template <int I>
    __device__ __forceinline__ void set(float a, float b) {
        if constexpr (sizeof(T) == 4 || N == 1) {
            w[I] = __builtin_bit_cast(uint32_t, a);
            if constexpr (N > 1) w[I + 1] = __builtin_bit_cast(uint32_t, b);
        } else if constexpr (__is_same(T, __bf16)) {
            w[I / 2] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
        } else {
            w[I / 2] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
        }
    }
};

// Cosine and sine of position * turns / 2^64 turns.  The product modulo 2^64 drops whole
// turns exactly (the frequency's rounding to 2^-64 turns is all that grows with the
// position): what is left is known to 2^-33 turns, and of that the nearest quarter is taken
// off as a whole number.  On an
// eighth of a turn either way (|t| <= pi/4) the power series up to t^9 and t^10 are off
// by less than 2^-28.
__device__ __forceinline__ void angle(int64_t position, uint64_t turns, float &c, float &s) {
    const uint64_t a = (uint64_t)position * turns;
    const uint32_t u = (uint32_t)((a + (1ull << 31)) >> 32) + (1u << 29);
    const uint32_t quarter = u >> 30;
    const float t = (float)((int32_t)(u & 0x3FFFFFFFu) - (1 << 29)) * 1.46291807926715968e-9f;
    const float z = t * t;
    float ss = __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040);
    ss = __builtin_fmaf(z, ss, 1.0f / 120);
    ss = __builtin_fmaf(z, ss, -1.0f / 6);
    ss = __builtin_fmaf(z * t, ss, t);
    float cc = __builtin_fmaf(z, -1.0f / 3628800, 1.0f / 40320);
    cc = __builtin_fmaf(z, cc, -1.0f / 720);
    cc = __builtin_fmaf(z, cc, 1.0f / 24);
    cc = __builtin_fmaf(z, cc, -0.5f);
    cc = __builtin_fmaf(z, cc, 1.0f);
    c = quarter & 1 ? ss : cc;
    s = quarter & 1 ? cc : ss;
    if ((quarter + 1) & 2) c = -c;
    if (quarter & 2) s = -s;
}

template <int N>
struct Angles {
    float c[N], s[N];
};

// Pairs I and I + 1 of N: in `a` the first channels, in `b` the second ones, or (NEXT)
// in `a` and then `b` the pairs one after the other.
template <typename T, int N, bool NEXT, int I = 0>
__device__ __forceinline__ void turn(Span<T, N> &a, Span<T, N> &b, const Angles<N> &g) {
    if constexpr (N == 1) {
        const float x = a.template get<0>(), y = b.template get<0>();
        a.template set<0>(__builtin_fmaf(x, g.c[0], -(y * g.s[0])), 0.0f);
        b.template set<0>(__builtin_fmaf(y, g.c[0], x * g.s[0]), 0.0f);
    } else if constexpr (I < N) {
        if constexpr (NEXT) {
            Span<T, N> &w = I < N / 2 ? a : b;
            constexpr int at = 2 * I % N;
            const float x = w.template get<at>(), y = w.template get<at + 1>();
            w.template set<at>(__builtin_fmaf(x, g.c[I], -(y * g.s[I])),
                               __builtin_fmaf(y, g.c[I], x * g.s[I]));
            turn<T, N, NEXT, I + 1>(a, b, g);
        } else {
            const float x0 = a.template get<I>(), y0 = b.template get<I>();
            const float x1 = a.template get<I + 1>(), y1 = b.template get<I + 1>();
            a.template set<I>(__builtin_fmaf(x0, g.c[I], -(y0 * g.s[I])),
                              __builtin_fmaf(x1, g.c[I + 1], -(y1 * g.s[I + 1])));
            b.template set<I>(__builtin_fmaf(y0, g.c[I], x0 * g.s[I]),
                              __builtin_fmaf(y1, g.c[I + 1], x1 * g.s[I + 1]));
            turn<T, N, NEXT, I + 2>(a, b, g);
        }
    }
}

// A thread takes one unit of a token's heads, every `lanes`-th of them: N pairs of
// channels whose angles it computes once, or 2N channels behind the turned ones, which
// are copied.  N = 16 bytes of channels, or 1 where sizes and strides do not allow it.
// Bound by memory: every channel is read once and written once.  Measured: 16001 tokens, 32
// and 8 heads of 128, bfloat16 (328 MB) 64 us, 5.1 TB/s (a large copy 4.8 to 5.4, by the
// card); 8190 tokens, 16 and 16 heads of 64, float32, 16 channels turned (134 MB) 25 us; 32
// tokens 4 us, a launch.
template <typename T, int N, bool NEXT>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryParams p) {
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (item >= p.items) return;
    const int unit = (int)(item % p.units);
    const int64_t rest = item / p.units;
    const int lane = (int)(rest % p.lanes);
    const int64_t token = rest / p.lanes;
    const bool copied = unit >= p.turned;
    // first channel of each half, and whether there is a second
    int at, step;
    bool both = true;
    if (copied) {
        at = p.rot + 2 * N * (unit - p.turned);
        step = N;
        both = at + N < p.dim;
    } else {
        at = NEXT ? 2 * N * unit : N * unit;
        step = NEXT ? N : p.rot / 2;
    }
    Angles<N> g;
    if (!copied) {
        const int64_t position = p.positions[token];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            angle(position, p.turns[N * unit + i], g.c[i], g.s[i]);
            g.c[i] *= p.factor;
            g.s[i] *= p.backward ? -p.factor : p.factor;
        }
    }
    const int heads = p.rows[0].heads + p.rows[1].heads;
    constexpr int kUnroll = 4;
    for (int h0 = lane; h0 < heads; h0 += kUnroll * p.lanes) {
        Span<T, N> a[kUnroll], b[kUnroll];
        T *to[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = h0 + u * p.lanes;
            if (h >= heads) continue;
            const bool second = h >= p.rows[0].heads;
            const Rows &r = p.rows[second];
            const int hh = second ? h - p.rows[0].heads : h;
            const T *x = (const T *)r.x + token * r.x_token + hh * r.x_head + at;
            to[u] = (T *)r.y + token * r.y_token + hh * r.y_head + at;
            a[u].load(x);
            if (both) b[u].load(x + step);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (h0 + u * p.lanes >= heads) continue;
            if (!copied) turn<T, N, NEXT>(a[u], b[u], g);
            a[u].store(to[u]);
            if (both) b[u].store(to[u] + step);
        }
    }
}

template <typename T, int N>
void launch(const RotaryParams &p, dim3 grid, hipStream_t s) {
    if (p.interleaved)
        hipLaunchKernelGGL((rotary_kernel<T, N, true>), grid, dim3(kThreads), 0, s, p);
    else
        hipLaunchKernelGGL((rotary_kernel<T, N, false>), grid, dim3(kThreads), 0, s, p);
}

lce_status validate_rows(const lce_rotary_rows *r, const char *name, int size) {
    if (r->heads < 1) return fail(LCE_EINVAL, "%s: heads %d must be >= 1", name, r->heads);
    if (!r->x || !r->y) return fail(LCE_EINVAL, "%s: x/y is NULL", name);
    if (!aligned(r->x, size) || !aligned(r->y, size))
        return fail(LCE_EALIGN, "%s: x and y must be aligned to their type", name);
    return LCE_OK;
}

// Rows of a tensor along one of its axes: how many, and how many elements apart.
struct Axis {
    int64_t count, apart;
};

lce_status validate_apart(const lce_rotary_rows *r, const char *name, int64_t tokens, int dim) {
    // rows that share memory would be written in any order, and in place read after that
    const Axis axes[2] = {{r->heads, std::abs(r->y_head_stride)}, {tokens, std::abs(r->y_token_stride)}};
    const Axis &in = axes[axes[1].apart < axes[0].apart], &out = axes[axes[1].apart >= axes[0].apart];
    if ((in.count > 1 && in.apart < dim) || (out.count > 1 && out.apart < dim) ||
        (in.count > 1 && out.count > 1 && (out.apart - dim) / (in.count - 1) < in.apart))
        return fail(LCE_EINVAL, "%s: rows of y overlap or lie between each other", name);
    if (r->x == r->y && ((r->heads > 1 && r->x_head_stride != r->y_head_stride) ||
                         (tokens > 1 && r->x_token_stride != r->y_token_stride)))
        return fail(LCE_EINVAL, "%s: y is x with other strides", name);
    return LCE_OK;
}

bool whole(const lce_rotary_rows &r, int per) {
    return aligned(r.x, 16) && aligned(r.y, 16) && r.x_token_stride % per == 0 &&
           r.x_head_stride % per == 0 && r.y_token_stride % per == 0 && r.y_head_stride % per == 0;
}

bool in_place(const lce_rotary_rows &r) {
    return r.x == r.y && r.x_token_stride == r.y_token_stride && r.x_head_stride == r.y_head_stride;
}

}  // namespace

extern "C" {

lce_status lce_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                                  double original, double *freqs, float *scale) {
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > 65536)
        return fail(LCE_EINVAL, "rot_dim %d is not an even number in [2, 65536]", rot_dim);
    if (!(base > 1.0) || !std::isfinite(base))
        return fail(LCE_EINVAL, "base %g is not a finite number > 1", base);
    if (scaling < LCE_ROTARY_PLAIN || scaling > LCE_ROTARY_YARN)
        return fail(LCE_EINVAL, "unknown scaling %d", scaling);
    if (scaling != LCE_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
        return fail(LCE_EINVAL, "factor %g is not a finite number >= 1", factor);
    // (the first pair turns once in 2 pi positions, and is the one that yarn leaves as it is)
    if (scaling == LCE_ROTARY_YARN && (!(original >= 7.0) || !std::isfinite(original)))
        return fail(LCE_EINVAL, "original %g is not a finite number >= 7", original);
    if (!freqs || !scale) return fail(LCE_EINVAL, "freqs/scale is NULL");
    const double r = rot_dim;
    if (scaling == LCE_ROTARY_NTK && rot_dim > 2) base *= std::pow(factor, r / (r - 2));
    if (!std::isfinite(base)) return fail(LCE_EINVAL, "base times a power of factor is infinite");
    // yarn: the pair numbers between which frequencies go from their own to slowed ones
    double first = 0, last = 1;
    if (scaling == LCE_ROTARY_YARN) {
        const double turn = 2 * M_PI;
        // (past r - 1 for both where every pair turns far more than 32 times: none is slowed)
        const auto number = [&](double turns) {
            return r * std::log(original / (turns * turn)) / (2 * std::log(base));
        };
        first = std::fmin(std::fmax(std::floor(number(32)), 0), r - 1);
        last = std::fmin(std::ceil(number(1)), r - 1);
        if (first == last) last += 0.001;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / r);
        freqs[i] = f;
        if (scaling == LCE_ROTARY_LINEAR) freqs[i] = f / factor;
        if (scaling == LCE_ROTARY_YARN) {
            const double m = std::fmin(std::fmax((i - first) / (last - first), 0), 1);
            freqs[i] = f / factor * m + f * (1 - m);
        }
    }
    *scale = scaling == LCE_ROTARY_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return ok();
}

lce_status lce_rotary_turns(const double *freqs, int32_t count, uint64_t *turns) {
    if (count < 1) return fail(LCE_EINVAL, "count %d must be >= 1", count);
    if (!freqs || !turns) return fail(LCE_EINVAL, "freqs/turns is NULL");
    for (int i = 0; i < count; ++i) {
        if (!std::isfinite(freqs[i])) return fail(LCE_EINVAL, "freqs[%d] is not finite", i);
        // 64 bits of mantissa: the fraction of a turn, to the nearest 2^-64 of its whole
        long double t = freqs[i] / 6.283185307179586476925286766559005768L;
        t -= std::floor(t);
        t = std::round(std::ldexp(t, 64));
        turns[i] = t >= 18446744073709551616.0L ? 0 : (uint64_t)t;
    }
    return ok();
}

lce_status lce_rotary(const lce_rotary_desc *desc, const uint64_t *turns, const int64_t *positions,
                      const lce_rotary_rows *q, const lce_rotary_rows *k, hipStream_t stream) {
    if (!desc) return fail(LCE_EINVAL, "desc is NULL");
    const lce_rotary_desc &d = *desc;
    if (d.tokens < 0) return fail(LCE_EINVAL, "tokens %d must be >= 0", d.tokens);
    if (d.head_dim < 2 || d.head_dim > 65536)
        return fail(LCE_EINVAL, "head_dim %d outside [2, 65536]", d.head_dim);
    if (d.rot_dim < 2 || d.rot_dim % 2 || d.rot_dim > d.head_dim)
        return fail(LCE_EINVAL, "rot_dim %d is not an even number in [2, %d]", d.rot_dim, d.head_dim);
    if (d.type != LCE_FLOAT32 && d.type != LCE_FLOAT16 && d.type != LCE_BFLOAT16)
        return fail(LCE_EINVAL, "unknown type %d", d.type);
    if ((d.interleaved != 0 && d.interleaved != 1) || (d.backward != 0 && d.backward != 1))
        return fail(LCE_EINVAL, "interleaved %d and backward %d must be 0 or 1", d.interleaved,
                    d.backward);
    if (!std::isfinite(d.scale)) return fail(LCE_EINVAL, "scale %g is not finite", d.scale);
    if (d.tokens == 0) return ok();
    if (!turns || !positions || !q) return fail(LCE_EINVAL, "turns/positions/q is NULL");
    if (!aligned(turns, 8) || !aligned(positions, 8))
        return fail(LCE_EALIGN, "turns and positions must be 8-byte aligned");
    const int size = d.type == LCE_FLOAT32 ? 4 : 2;
    if (const lce_status st = validate_rows(q, "q", size)) return st;
    if (k)
        if (const lce_status st = validate_rows(k, "k", size)) return st;

    // 16 bytes at a time where pairs, copied channels, addresses and strides allow it
    const int wide = 16 / size;
    const bool fits = d.rot_dim % (2 * wide) == 0 && d.head_dim % wide == 0 && whole(*q, wide) &&
                      (!k || whole(*k, wide));
    const int n = fits ? wide : 1;
    RotaryParams p;
    p.rows[0] = Rows{q->x, q->y, q->x_token_stride, q->x_head_stride, q->y_token_stride,
                     q->y_head_stride, q->heads};
    p.rows[1] = k ? Rows{k->x, k->y, k->x_token_stride, k->x_head_stride, k->y_token_stride,
                         k->y_head_stride, k->heads}
                  : Rows{};
    p.turns = turns, p.positions = positions;
    p.dim = d.head_dim, p.rot = d.rot_dim, p.interleaved = d.interleaved, p.backward = d.backward;
    p.factor = d.scale;
    p.turned = d.rot_dim / 2 / n;
    const bool stay = in_place(*q) && (!k || in_place(*k));   // nothing to copy
    p.units = p.turned + (stay ? 0 : (d.head_dim - d.rot_dim + 2 * n - 1) / (2 * n));
    const int64_t heads = (int64_t)q->heads + (k ? k->heads : 0);
    if (heads > 1 << 20) return fail(LCE_EUNSUPPORTED, "%lld heads: too many", (long long)heads);
    // threads that share a token's heads: as many as there are heads where the call is
    // short, fewer (and angles computed less often) once that is enough threads
    // (the product with all heads can pass 64 bits)
    const int64_t each = (int64_t)d.tokens * p.units;
    int64_t lanes = heads;
    while (lanes > 1 && each > 256 * 2048 / lanes) lanes = (lanes + 1) / 2;
    p.lanes = (int)lanes;
    p.items = each * lanes;
    const int64_t groups = (p.items + kThreads - 1) / kThreads;
    if (groups > (1 << 24) - 1)
        return fail(LCE_EUNSUPPORTED, "%d tokens of %lld heads: too many for one call", d.tokens,
                    (long long)heads);
    if (const lce_status st = validate_apart(q, "q", d.tokens, d.head_dim)) return st;
    if (k) {
        if (const lce_status st = validate_apart(k, "k", d.tokens, d.head_dim)) return st;
        // either's results would be written over the other's, or over what it still reads
        if (q->y == k->y || q->y == k->x || k->y == q->x)
            return fail(LCE_EINVAL, "q and k: y of one is x or y of the other");
    }
    const dim3 grid((unsigned)groups);
    if (d.type == LCE_FLOAT32)
        n > 1 ? launch<float, 4>(p, grid, stream) : launch<float, 1>(p, grid, stream);
    else if (d.type == LCE_FLOAT16)
        n > 1 ? launch<_Float16, 8>(p, grid, stream) : launch<_Float16, 1>(p, grid, stream);
    else
        n > 1 ? launch<__bf16, 8>(p, grid, stream) : launch<__bf16, 1>(p, grid, stream);
    return check_launch("lce_rotary launch");
}

}  // extern "C"
