// The 4-bit key/value cache: record layout (the one that lce.h gives) and the
// device helpers that its kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lce.h"

namespace lce {
namespace kv4 {

constexpr int kPage = LCE_KV4_PAGE;
constexpr int kThreads = 256;
// Tickets are 64 bytes apart: draws from one line of memory wait for each other.
constexpr int kTicketStride = 16;
constexpr int kTickets = LCE_KV4_WORKSPACE_ZERO / (4 * kTicketStride);

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

// Byte offsets of a record's parts, for a head of D channels.
template <int D>
struct Record {
    static constexpr int kKey = 0;
    static constexpr int kValue = 32 * D;
    static constexpr int kKeyScale = 64 * D;
    static constexpr int kValueScale = 66 * D;
    static constexpr int kSigns = 68 * D;
    static constexpr int kBytes = 76 * D;
};

template <typename A, typename B>
__device__ __forceinline__ A bits_as(const B &b) {
    static_assert(sizeof(A) == sizeof(B), "same size");
    return __builtin_bit_cast(A, b);
}

// The float whose exponent field is the byte: what the conversions to and
// from e2m1 take as their scale (they look at nothing else of it; 0 is 2^-127,
// 255 is NaN).
__device__ __forceinline__ float scale_of(uint32_t byte) { return bits_as<float>(byte << 23); }

// Reductions over the four lanes l, l^16, l^32, l^48 (the rows of a wave of
// 64): both swaps return each lane's own value and its partner's.
template <typename F>
__device__ __forceinline__ float across_rows(float x, F f) {
    const uint32_t u = bits_as<uint32_t>(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float y = f(bits_as<float>((uint32_t)a[0]), bits_as<float>((uint32_t)a[1]));
    const uint32_t w = bits_as<uint32_t>(y);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return f(bits_as<float>((uint32_t)b[0]), bits_as<float>((uint32_t)b[1]));
}

// Below every score, and finite: a row that has seen nothing yet weighs a hidden
// token exp2(-infinity - kNone) = 0.
constexpr float kNone = -3.402823466e38f;

// Scores (log2) up to which half a last place is at most a half, 2^kLag more included.
constexpr float kLarge = 8388608.0f;

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// One sequence of a batch, as the device arrays give it; every value is
// forced into its range, so that no index computed from it leaves a buffer.
struct Sequence {
    int index;    // -1: none
    int start;    // first query token
    int queries;
    int length;   // cached tokens, 0 .. 64*width
};

// The last sequence b whose first work item is at or before `item` (uniform
// over the wave; all 64 lanes take part).  Items of b begin at
// first(clamped q_start[b], b), which does not fall as b grows.
template <typename First>
__device__ __forceinline__ Sequence find_sequence(const int32_t *q_start, const int32_t *lengths,
                                                  int seqs, int tokens, int width, int64_t item,
                                                  First first) {
    const int lane = threadIdx.x & 63;
    Sequence s;
    s.index = -1;
    s.start = s.queries = s.length = 0;
    for (int base = 0; base < seqs; base += 64) {
        // everything a sequence has, one a lane, in one round trip to memory
        const int b = min(base + lane, seqs - 1);
        const int start = clampi(q_start[b], 0, tokens), end = clampi(q_start[b + 1], 0, tokens);
        const int length = lengths[b];
        const uint64_t mask =
            __builtin_amdgcn_ballot_w64(base + lane < seqs && first(start, b) <= item);
        if (mask) {
            const int at = 63 - __builtin_clzll(mask);
            s.index = base + at;
            s.start = __builtin_amdgcn_readlane(start, at);
            s.queries = max(__builtin_amdgcn_readlane(end, at) - s.start, 0);
            s.length = (int)min(max((int64_t)__builtin_amdgcn_readlane(length, at), (int64_t)0),
                                (int64_t)kPage * width);
        }
        if (mask != ~0ull) break;
    }
    return s;
}

// Visible tokens [lo, hi) of query i of a sequence.
struct Span {
    int lo, hi;
};

__device__ __forceinline__ Span visible(const Sequence &s, int i, int causal, int window) {
    const int p = s.length - s.queries + i;
    Span v;
    v.hi = causal ? clampi(p + 1, 0, s.length) : s.length;
    v.lo = window > 0 ? (int)min(max((int64_t)p - window + 1, (int64_t)0), (int64_t)s.length) : 0;
    return v;
}

}  // namespace kv4
}  // namespace lce
