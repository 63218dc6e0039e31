// The 8-bit key/value cache: record layout (the one that lce.h gives), parameters and
// launchers of its kernels.  The C ABI in kv8.hip checks a call and plans it, and calls
// one of these.  Element types, sequences and the joining of splits are the 4-bit cache's.
#pragma once

#include "kv4_attend.hpp"

namespace lce {
namespace kv8 {

using namespace kv4;

constexpr int kBlock = LCE_KV8_BLOCK;     // tokens that share a scale
constexpr int kBlocks = kPage / kBlock;

// Byte offsets of a record's parts, for a head of D channels.
template <int D>
struct Record {
    static constexpr int kKey = 0;              // [token][D]
    static constexpr int kValue = 64 * D;       // [token / 4][D][token % 4]
    static constexpr int kScale = 128 * D;      // of the keys' blocks, of the values'
    static constexpr int kBytes = 128 * D + 128;
};

// Scales that hold a finite float32: the smallest normal power of two to that of
// 448 * 2^120.
constexpr int kLeastScale = 1, kMostScale = 247;

struct AppendParams {
    uint8_t *cache;
    const void *k, *v;
    const int32_t *table, *q_start, *lengths;
    int64_t k_token, k_head, v_token, v_head;   // strides in elements
    int64_t items;                              // blocks * kv_heads
    int pages, kv_heads, tokens, seqs, width;
};

struct ReadParams {
    const uint8_t *cache;
    const int64_t *slots;
    void *k, *v;
    int64_t tokens;
    int pages, kv_heads;
};

// A call's query tokens over cached sequences.
struct AttendParams {
    const uint8_t *cache;
    const void *q;
    const int32_t *table, *q_start, *lengths;
    const int32_t *prefix;                               // or null
    const float *slopes;                                 // or null
    void *out;
    float *lse;                                          // or null
    int32_t *tickets;                                    // workspace: one per shared unit
    float *part;                                         // workspace: partial results
    int64_t q_token, q_head;                             // strides in elements
    float scale_log2;
    float cap_log2, cap_inverse;                         // of scores, or 0; 1 / cap_log2
    int pages, kv_heads, group;                          // group = q_heads / kv_heads
    int tokens, seqs, width, causal, window;
    int chunk;                                           // pages per workgroup
    int turn;                                            // grid width if splits turn, or 0
};

// Visible tokens of query i of a sequence, `prefix` of which every query sees that the
// window leaves.
__device__ __forceinline__ Span visible(const Sequence &s, int i, int causal, int window,
                                        int prefix) {
    const int p = s.length - s.queries + i;
    Span v;
    v.hi = causal ? clampi(max(p + 1, prefix), 0, s.length) : s.length;
    v.lo = window > 0 ? (int)min(max((int64_t)p - window + 1, (int64_t)0), (int64_t)s.length) : 0;
    return v;
}

void launch_append(const AppendParams &p, int type, int dim, hipStream_t s);
void launch_read(const ReadParams &p, int type, int dim, hipStream_t s);
// 16 or 32 query rows a workgroup; grid = (tiles * kv_heads, splits); few: rows of a sequence
// and head; once (of few): loads past the caches
void launch_attend16(const AttendParams &p, int type, int dim, int rows, bool few, bool once,
                     dim3 grid, hipStream_t s);
// 128 query rows a workgroup, heads of up to 128; grid = (tiles * kv_heads, splits)
void launch_attend128(const AttendParams &p, int type, int dim, dim3 grid, hipStream_t s);

}  // namespace kv8
}  // namespace lce
