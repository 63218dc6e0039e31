// Parameters and launchers of the 4-bit cache's kernels: the C ABI in kv4.hip
// checks a call and plans it, and calls one of these.
#pragma once

#include "kv4.hpp"

namespace lce {
namespace kv4 {

struct AppendParams {
    uint8_t *cache;
    const void *k, *v;
    const int64_t *slots;
    int64_t tokens, k_token, k_head, v_token, v_head;   // strides in elements
    int pages, kv_heads;
};

struct ReadParams {
    const uint8_t *cache;
    const int64_t *slots;
    void *k, *v;
    int64_t tokens;
    int pages, kv_heads;
};

// A call's query tokens over cached sequences.
struct QueryParams {
    const uint8_t *cache;
    const void *q;
    const int32_t *table, *q_start, *lengths;
    int64_t q_token, q_head;                             // strides in elements
    int pages, kv_heads, group;                          // group = q_heads / kv_heads
    int tokens, seqs, width, causal, window, list;
    int chunk;                                           // pages per workgroup
    int32_t *tickets;                                    // workspace: one per shared unit
};

struct AttendParams : QueryParams {
    const int32_t *named;                                // list of pages, or null
    void *out;
    float *lse;                                          // or null
    float *part;                                         // workspace: partial results
    float scale_log2;
    int turn;                                            // grid width if splits turn, or 0
};

struct SelectParams : QueryParams {
    int keep_first, keep_last;
    int32_t *chosen;
    uint16_t *ranks;                                     // workspace: [token][head][width]
};

void launch_append(const AppendParams &p, int type, int dim, hipStream_t s);
void launch_read(const ReadParams &p, int type, int dim, hipStream_t s);
// 16 or 32 query rows a workgroup (32: heads of up to 128); grid = (tiles *
// kv_heads, splits); once: heads of 128 are loaded past the caches
void launch_attend16(const AttendParams &p, int type, int dim, int rows, bool once, dim3 grid,
                     hipStream_t s);
// 128 query rows a workgroup, no list; grid = (tiles * kv_heads, splits)
void launch_attend128(const AttendParams &p, int type, int dim, dim3 grid, hipStream_t s);
// one token and head of the cache a workgroup; grid = (tokens * kv_heads, splits)
void launch_select(const SelectParams &p, int type, int dim, dim3 grid, hipStream_t s);

}  // namespace kv4
}  // namespace lce
