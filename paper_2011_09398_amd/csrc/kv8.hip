// C ABI of the 8-bit key/value cache (declared in lce.h): host-side checks and the split
// of the work.  No allocation, no synchronization.
#include <algorithm>
#include <cmath>

#include "kv8.hpp"
#include "status.hpp"

namespace {

using lce::aligned;
using lce::check_launch;
using lce::fail;
using lce::ok;
using lce::tuning;
using lce::kv8::kBlock;
using lce::kv8::kPage;

constexpr double kCus = 256;
// Workgroups of 256 threads in a grid: threads are counted in 32 bits.
constexpr int64_t kMostGroups = (1LL << 24) - 1;

lce_status validate_cache(const lce_kv8_cache_desc *d) {
    if (!d) return fail(LCE_EINVAL, "desc is NULL");
    if (d->pages < 1 || d->kv_heads < 1)
        return fail(LCE_EINVAL, "pages %d and kv_heads %d must be >= 1", d->pages, d->kv_heads);
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
        return fail(LCE_EUNSUPPORTED, "head_dim %d is not 64, 128 or 256", d->head_dim);
    if (d->kv_heads > 65535)
        return fail(LCE_EUNSUPPORTED, "kv_heads %d exceeds 65535", d->kv_heads);
    return LCE_OK;
}

lce_status validate_sequences(int32_t seqs, int32_t width) {
    if (seqs < 1 || width < 1)
        return fail(LCE_EINVAL, "seqs %d and table_width %d must be >= 1", seqs, width);
    if (width > 1 << 24)
        return fail(LCE_EUNSUPPORTED, "table_width %d: sequences of more than 2^30 tokens", width);
    return LCE_OK;
}

lce_status validate_type(int32_t type) {
    if (type != LCE_FLOAT32 && type != LCE_FLOAT16 && type != LCE_BFLOAT16)
        return fail(LCE_EINVAL, "unknown type %d", type);
    return LCE_OK;
}

lce_status validate_query(const lce_kv8_cache_desc *d, const lce_kv8_query_desc *q) {
    if (const lce_status st = validate_cache(d)) return st;
    if (!q) return fail(LCE_EINVAL, "query is NULL");
    if (q->tokens < 0) return fail(LCE_EINVAL, "tokens %d must be >= 0", q->tokens);
    if (const lce_status st = validate_sequences(q->seqs, q->table_width)) return st;
    if (q->q_heads < 1 || q->q_heads % d->kv_heads)
        return fail(LCE_EINVAL, "q_heads %d is not a multiple of kv_heads %d", q->q_heads,
                    d->kv_heads);
    // rows and workgroups are counted in 32 bits
    if (((int64_t)q->tokens + q->seqs) * q->q_heads > INT32_MAX)
        return fail(LCE_EUNSUPPORTED, "%d tokens of %d heads in %d sequences: too many for one call",
                    q->tokens, q->q_heads, q->seqs);
    return LCE_OK;
}

lce_status validate_call(const lce_kv8_cache_desc *d, const lce_kv8_query_desc *q) {
    if (const lce_status st = validate_query(d, q)) return st;
    if (q->type != LCE_FLOAT16 && q->type != LCE_BFLOAT16)
        return fail(q->type == LCE_FLOAT32 ? LCE_EUNSUPPORTED : LCE_EINVAL,
                    "query type %d is not float16 or bfloat16", q->type);
    if (q->causal != 0 && q->causal != 1) return fail(LCE_EINVAL, "causal %d is not 0 or 1", q->causal);
    if (q->window < 0 || q->max_q < 0 || q->max_len < 0)
        return fail(LCE_EINVAL, "window %d, max_q %d and max_len %d must be >= 0", q->window,
                    q->max_q, q->max_len);
    if (!(q->scale > 0.0f) || !std::isfinite(q->scale * 1.44269504088896341f))
        return fail(LCE_EINVAL, "scale %g is not a finite number > 0", q->scale);
    if (q->softcap != 0.0f && !(q->softcap >= 1e-30f && q->softcap <= 1e30f))
        return fail(LCE_EINVAL, "softcap %g is not 0 or in [1e-30, 1e30]", q->softcap);
    return LCE_OK;
}

// What the workspace has room for: states of this many tiles of 16 rows, an eighth
// of it of 128.  More workgroups would not run at the same time anyway.
constexpr int64_t kMostParts = 4096;
static_assert(kMostParts / 2 <= lce::kv4::kTickets, "a ticket for each unit that is shared");

// Tiles of `rows` query rows of a cache head.
int64_t tiles(const lce_kv8_cache_desc &d, const lce_kv8_query_desc &q, int rows) {
    return (int64_t)q.tokens * (q.q_heads / d.kv_heads) / rows + q.seqs;
}

// Pages that a tile can have before it, as far as the call says.
int64_t most_pages(const lce_kv8_query_desc &q, bool prefix) {
    int64_t n = q.table_width;
    if (q.max_len > 0) n = std::min<int64_t>(n, (q.max_len + (int64_t)kPage - 1) / kPage);
    if (q.window > 0 && q.causal && !prefix)
        n = std::min<int64_t>(n, ((int64_t)q.window + std::max(q.max_q, 1)) / kPage + 2);
    return n;
}

// The most rows that read the same pages, as far as the call says: the new tokens of a
// sequence times the heads that share a cache head.
int64_t query_rows(const lce_kv8_cache_desc &d, const lce_kv8_query_desc &q) {
    return (q.max_q > 0 ? q.max_q : ((int64_t)q.tokens + q.seqs - 1) / q.seqs) *
           (q.q_heads / d.kv_heads);
}

// Query rows of a tile.  In tiles of 128 rows a page's codes become two-byte floats once
// for all of them, but the more rows a tile has the fewer tiles there are, and fewer than run
// at a time (512) leave CUs without work; tiles of 16 and 32 rows share a page between their
// rows alone, and their waves share the pages.  Heads of 64 channels have half the products
// for the same softmax, which the smaller tiles' third wave a SIMD does better, until there
// are many tiles.  Heads of 256 channels stay at 16: 32 rows of them, or 128, have more state
// than the registers of two waves a SIMD (one wave a SIMD is not tried).  The rule is short and
// not the least of every line: 16 sequences of 64 new tokens take 32 rows, for 15 to 31 % more
// time than 16, and the last line's prompts of 128 channels 128 rows, for 8 to 26 % more than
// 32.  Measured in graphs (us, tiles of 16 / 32 / 128; 32 heads on 8 if not said
// otherwise; the last two columns float16):
//                                          128 channels      64 channels      128, capped
//   16 of 4064 tokens, 64 of them new      48 / 55 / 99      29 / 38 / 80     54 / 65 / 130
//   one of 5024, 1024 new                 142 / 111 / 121    81 / 65 / 97    158 / 130 / 157
//   one of 6048, 2048 new                 279 / 222 / 183   162 / 123 / 129  324 / 274 / 238
//   one of 8096, 4096 new                 640 / 512 / 413   366 / 277 / 286  767 / 627 / 531
//   four of up to 4512, up to 512 new      86 / 75 / 111     52 / 41 / 89    98 / 88 / 146
//   four of up to 5024, up to 1024 new    166 / 137 / 126   101 / 76 / 100   190 / 165 / 162
//   four of up to 6048, up to 2048 new    330 / 272 / 206   197 / 149 / 145  390 / 325 / 269
//   16 of up to 1024, up to 128 new        34 / 34 / 33      25 / 22 / 26     36 / 37 / 43
//   one prompt of 1024                     29 / 28 / 31      21 / 20 / 25     33 / 32 / 41
//   one prompt of 2048                     81 / 71 / 61      50 / 40 / 47     91 / 80 / 80
//   two of up to 5025, 359 new, 8 on 2     30 / 31 / 60      18 / 20 / 40     32 / 36 / 67
//   four prompts of up to 1943, 2 on 1     19 / 23 / 49      12 / 16 / 31     20 / 26 / 51
//   three prompts of up to 2500, 16 on 2   66 / 62 / 67      45 / 37 / 54     78 / 70 / 88
int tile_rows(const lce_kv8_cache_desc &d, const lce_kv8_query_desc &q) {
    if (d.head_dim > 128) return 16;
    const int forced = tuning(LCE_TUNE_KV8_ROWS);
    if (forced == 16 || forced == 32 || forced == 128) return forced;
    const int64_t most = query_rows(d, q), all = (int64_t)q.tokens * q.q_heads;
    if (most >= 128 && all >= 128 * (d.head_dim == 64 ? 2048 : 512)) return 128;
    return most >= 256 && all >= 32 * 1024 ? 32 : 16;
}

// Most states of one tile, of `units` tiles with room for `parts` states.
int64_t most_splits(int64_t units, int64_t parts) {
    return std::min<int64_t>(std::max<int64_t>(parts / std::max<int64_t>(units, 1), 1),
                             lce::kv4::kMostSplits);
}

// What states take: with each height of a tile, up to a table's pages of them for each,
// or as many as there is room for.  More tokens never take less, so that a workspace
// serves calls with fewer, too.
int64_t state_bytes(const lce_kv8_cache_desc &d, const lce_kv8_query_desc &q) {
    const int64_t splits = std::min<int64_t>(q.table_width, lce::kv4::kMostSplits);
    if (splits < 2 || q.tokens == 0) return 0;
    int64_t most = 0;
    for (const int rows : {16, 32, 128}) {
        const int64_t units = tiles(d, q, rows) * d.kv_heads;
        most = std::max(most, std::min(kMostParts * 16 / rows, units * splits) * rows);
    }
    return most * (d.head_dim + 4) * 4;
}

struct Split {
    int chunk;    // pages per workgroup
    int splits;   // workgroups that share a tile, at most
};

// What a tile's pages cost and what sharing it does, in microseconds: `step` for a wave to
// take a page, `fixed` for the partial states, the ticket and the joining, and `each` for
// every state joined, which one workgroup reads.
struct Cost {
    double step, fixed, each;
};

// `pages` pages of each of `likely` tiles (the grid has room for `units`): how many
// workgroups (of four waves) share a tile.  It is divided only where its pages take longer,
// and no further than `most` workgroups in all and `parts` states in the workspace; the
// number of pages that a workgroup takes is a multiple of `whole`, so that all waves are
// busy to the end.  Windows span `usual` pages, one or two less than they can.
Split split_pages(int64_t units, int64_t likely, int64_t pages, int64_t usual, const Cost &c,
                  int64_t most, int64_t parts, int64_t whole) {
    const double some = (double)std::max<int64_t>(likely, 1);
    const int64_t room = most_splits(units, parts);
    int64_t chunk = std::max<int64_t>(pages, 1);
    if (const int t = tuning(LCE_TUNE_KV8_CHUNK)) {
        chunk = std::clamp<int64_t>(t, 1, chunk);
    } else {
        const double alone = usual * c.step / 4;
        // the least of alone / z + fixed + each * z
        double z = std::min(std::min((double)room, (double)most / some), std::sqrt(alone / c.each));
        // (one workgroup a CU, rather than two on some)
        if (z * some > kCus && z * some < 2 * kCus) z = std::max(kCus / some, 1.0);
        if (z > 1 && alone / z + c.fixed + c.each * z < alone)
            chunk = ((int64_t)std::ceil(usual / z) + whole - 1) / whole * whole;
    }
    // (more pages than usual could be more states than there is room for)
    chunk = std::max(chunk, (pages + room - 1) / room);
    Split s;
    s.chunk = (int)chunk;
    s.splits = (int)std::max<int64_t>((pages + chunk - 1) / chunk, 1);
    return s;
}

}  // namespace

extern "C" {

lce_status lce_kv8_cache_size(const lce_kv8_cache_desc *desc, int64_t *bytes) {
    if (!bytes) return fail(LCE_EINVAL, "bytes output pointer is NULL");
    if (const lce_status st = validate_cache(desc)) return st;
    *bytes = (int64_t)desc->pages * desc->kv_heads * 128 * (desc->head_dim + 1);
    return ok();
}

lce_status lce_kv8_append(const lce_kv8_cache_desc *desc, void *cache, int32_t type,
                          const void *k, int64_t k_token_stride, int64_t k_head_stride,
                          const void *v, int64_t v_token_stride, int64_t v_head_stride,
                          int32_t tokens, int32_t seqs, int32_t table_width, const int32_t *table,
                          const int32_t *q_start, const int32_t *lengths, hipStream_t stream) {
    if (const lce_status st = validate_cache(desc)) return st;
    if (const lce_status st = validate_type(type)) return st;
    if (tokens < 0) return fail(LCE_EINVAL, "tokens %d must be >= 0", tokens);
    if (const lce_status st = validate_sequences(seqs, table_width)) return st;
    // a sequence's n new tokens touch at most floor(n / 16) + 2 blocks
    const int64_t items = ((int64_t)tokens / kBlock + 2 * (int64_t)seqs) * desc->kv_heads;
    if (items / 4 >= kMostGroups)
        return fail(LCE_EUNSUPPORTED, "%d tokens of %d heads in %d sequences: too many for one call",
                    tokens, desc->kv_heads, seqs);
    if (tokens == 0) return ok();
    if (!cache || !k || !v || !table || !q_start || !lengths)
        return fail(LCE_EINVAL, "cache/k/v/table/q_start/lengths is NULL");
    if (!aligned(cache, 16) || !aligned(k, 16) || !aligned(v, 16))
        return fail(LCE_EALIGN, "cache, k and v must be 16-byte aligned");
    if (!aligned(table, 4) || !aligned(q_start, 4) || !aligned(lengths, 4))
        return fail(LCE_EALIGN, "table, q_start and lengths must be 4-byte aligned");
    const int64_t unit = type == LCE_FLOAT32 ? 4 : 8;
    if (k_token_stride % unit || k_head_stride % unit || v_token_stride % unit ||
        v_head_stride % unit)
        return fail(LCE_EALIGN, "strides must be multiples of 16 bytes (%lld elements)",
                    (long long)unit);
    lce::kv8::AppendParams p;
    p.cache = static_cast<uint8_t *>(cache);
    p.k = k, p.v = v;
    p.table = table, p.q_start = q_start, p.lengths = lengths;
    p.k_token = k_token_stride, p.k_head = k_head_stride;
    p.v_token = v_token_stride, p.v_head = v_head_stride;
    p.items = items;
    p.pages = desc->pages, p.kv_heads = desc->kv_heads;
    p.tokens = tokens, p.seqs = seqs, p.width = table_width;
    lce::kv8::launch_append(p, type, desc->head_dim, stream);
    return check_launch("lce_kv8_append launch");
}

lce_status lce_kv8_read(const lce_kv8_cache_desc *desc, const void *cache, const int64_t *slots,
                        int64_t tokens, int32_t type, void *k, void *v, hipStream_t stream) {
    if (const lce_status st = validate_cache(desc)) return st;
    if (const lce_status st = validate_type(type)) return st;
    if (tokens < 0 || tokens > INT32_MAX)
        return fail(LCE_EINVAL, "tokens %lld outside [0, 2^31)", (long long)tokens);
    // workgroups of at least 8 tokens of one head
    if ((tokens / 8 + 1) * desc->kv_heads > kMostGroups)
        return fail(LCE_EUNSUPPORTED, "%lld tokens of %d heads: too many for one call",
                    (long long)tokens, desc->kv_heads);
    if (tokens == 0) return ok();
    if (!cache || !k || !v || !slots) return fail(LCE_EINVAL, "cache/k/v/slots is NULL");
    if (!aligned(cache, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8))
        return fail(LCE_EALIGN, "cache, k and v must be 16-byte aligned, slots 8-byte");
    lce::kv8::ReadParams p;
    p.cache = static_cast<const uint8_t *>(cache);
    p.slots = slots, p.k = k, p.v = v, p.tokens = tokens;
    p.pages = desc->pages, p.kv_heads = desc->kv_heads;
    lce::kv8::launch_read(p, type, desc->head_dim, stream);
    return check_launch("lce_kv8_read launch");
}

lce_status lce_kv8_workspace_size(const lce_kv8_cache_desc *desc, const lce_kv8_query_desc *query,
                                  int64_t *bytes) {
    if (!bytes) return fail(LCE_EINVAL, "bytes output pointer is NULL");
    if (const lce_status st = validate_query(desc, query)) return st;
    *bytes = LCE_KV8_WORKSPACE_ZERO + state_bytes(*desc, *query);
    return ok();
}

lce_status lce_kv8_attention(const lce_kv8_cache_desc *desc, const void *cache,
                             const lce_kv8_query_desc *query, const void *q, const int32_t *table,
                             const int32_t *q_start, const int32_t *lengths, const float *slopes,
                             const int32_t *prefix, void *out, float *lse, void *workspace,
                             int64_t workspace_bytes, hipStream_t stream) {
    if (const lce_status st = validate_call(desc, query)) return st;
    if (query->tokens == 0) return ok();
    if (!cache || !q || !table || !q_start || !lengths || !out || !workspace)
        return fail(LCE_EINVAL, "cache/q/table/q_start/lengths/out/workspace is NULL");
    if (!aligned(cache, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16))
        return fail(LCE_EALIGN, "cache, q, out and workspace must be 16-byte aligned");
    if (!aligned(table, 4) || !aligned(q_start, 4) || !aligned(lengths, 4) || !aligned(slopes, 4) ||
        !aligned(prefix, 4) || !aligned(lse, 4))
        return fail(LCE_EALIGN,
                    "table, q_start, lengths, slopes, prefix and lse must be 4-byte aligned");
    if (query->q_token_stride % 8 || query->q_head_stride % 8)
        return fail(LCE_EALIGN, "q strides must be multiples of 8 elements");
    int64_t need = 0;
    if (const lce_status st = lce_kv8_workspace_size(desc, query, &need)) return st;
    if (workspace_bytes < need)
        return fail(LCE_EINVAL, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                    (long long)need);

    const int rows = tile_rows(*desc, *query);
    const int64_t units = tiles(*desc, *query, rows) * desc->kv_heads;
    const double size = desc->head_dim / 128.0;
    const int64_t slots = desc->head_dim > 128 ? 512 : 768;   // workgroups that run at a time
    const int64_t most = most_pages(*query, prefix != nullptr);
    const int64_t each = query_rows(*desc, *query);
    const bool several = each > 64;
    // the grid has a tile to spare for each sequence; most calls have fewer (counted in
    // floating point: max_q is the caller's word)
    const double spread = query->seqs * (double)desc->kv_heads;
    const int64_t likely = (int64_t)std::min((double)units, spread * ((each + rows - 1) / rows));
    // Where no window makes sequences alike and there are fewer tiles than run at a time, up
    // to four times as many workgroups as do: sequences are of different lengths, of which
    // the call knows the longest.  Measured in graphs over three caches (us by pages a
    // workgroup; one new token and 32 heads on 8 of 128 channels if not said otherwise):
    //                                         choice    8    12    16    24    32    64   all
    //   1 of 30011                              18.9  23.0  20.9  18.9  20.4  22.6  34.9   205
    //   48 of up to 8192                        58.8  58.7  58.8  58.9  59.5  59.3     -  81.7
    //   16, window 4096, 4 new, 16 on 8 of 256  44.9  51.1  53.4  45.0  49.4  55.9     -  66.7
    //   24 of up to 4001, 32 on 32 of 64        36.5  43.1  42.5  41.2  39.0  39.8     -  38.8
    //   27 of up to 3877, 4 new, 4 on 1 of 256  22.6  22.6  25.4  27.2  32.9  38.9  54.9  54.7
    //   14 of up to 11385, 5, 10 on 2 of 256    37.0  46.0  37.2  36.9  37.6  41.3  56.1   122
    //   2 of up to 26367, 16 on 4 of 256        25.2  27.4  26.6  25.3  30.2  34.9  58.3   320
    //   26 of up to 7976, 8 on 2                17.6  17.6  20.2  19.5  23.5  26.1  44.1  76.4
    //   4 of up to 33362, 64 on 4 of 64         23.8  30.5  23.0  22.6  23.7  23.4  28.5   167
    //   29 of up to 2315, 128 on 8 of 64        21.8  21.7  20.6  19.0  21.1  24.1  23.6  23.6
    const int64_t usual =
        most < most_pages(*query, true) ? std::max<int64_t>(most - 2, 1) : most;
    // kB of a tile's state: a workgroup writes them at 5, and the last one reads 45 a us
    const double state = std::min<int64_t>(each, rows) * desc->head_dim * 4e-3;
    const Cost cost = rows == 128 ? Cost{2 + 2 * size, 4 + 8 * size, 0.06}
                                  : Cost{0.3 + size, (1.2 + state * 0.19) * (several ? 2.0 : 1.0),
                                         0.05 + state / 45};
    const int64_t limit = rows == 128 || several ? 512
                          : query->window        ? slots
                          : likely < slots       ? 4 * slots
                                                 : 7 * slots / 4;
    const Split s = split_pages(units, likely, most, usual, cost, limit, kMostParts * 16 / rows,
                                rows == 128 ? 1 : 4);
    // Loads past the caches where no other tile reads the same pages and the whole is long
    // (all sequences as long as the longest: calls read half of that or less): 48 of up to
    // 8192 tokens 59 us against 64 through them.
    const bool once = each <= 16 && 128.0 * desc->head_dim * most * likely >= (240 << 20);
    lce::kv8::AttendParams p;
    p.cache = static_cast<const uint8_t *>(cache);
    p.q = q;
    p.table = table, p.q_start = q_start, p.lengths = lengths;
    p.prefix = query->causal ? prefix : nullptr;
    p.slopes = slopes;
    p.out = out, p.lse = lse;
    p.tickets = static_cast<int32_t *>(workspace);
    p.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + LCE_KV8_WORKSPACE_ZERO);
    p.q_token = query->q_token_stride, p.q_head = query->q_head_stride;
    p.scale_log2 = query->scale * 1.44269504088896341f;
    p.cap_log2 = query->softcap * 1.44269504088896341f;
    p.cap_inverse = p.cap_log2 > 0.0f ? 1.0f / p.cap_log2 : 0.0f;
    p.pages = desc->pages, p.kv_heads = desc->kv_heads, p.group = query->q_heads / desc->kv_heads;
    p.tokens = query->tokens, p.seqs = query->seqs, p.width = query->table_width;
    p.causal = query->causal, p.window = query->window;
    p.chunk = s.chunk;
    p.turn = units % 8 == 0 && desc->kv_heads % 8 ? (int)units : 0;
    if (units > kMostGroups)
        return fail(LCE_EUNSUPPORTED, "%lld tiles: too many for one call", (long long)units);
    const dim3 grid((unsigned)units, (unsigned)s.splits);
    static const char *const kNames[2][3] = {
        {"kv8-16", "kv8-32", "kv8-128"}, {"kv8-16-split", "kv8-32-split", "kv8-128-split"}};
    lce::g_last_schedule = kNames[s.splits > 1][rows == 16 ? 0 : rows == 32 ? 1 : 2];
    if (rows == 128)
        lce::kv8::launch_attend128(p, query->type, desc->head_dim, grid, stream);
    else
        lce::kv8::launch_attend16(p, query->type, desc->head_dim, rows, !several, once, grid,
                                   stream);
    return check_launch("lce_kv8_attention launch");
}

}  // extern "C"
