// C ABI of the 4-bit key/value cache (declared in lce.h): host-side checks and
// the split of the work.  No allocation, no synchronization.
#include <algorithm>
#include <cmath>

#include "kv4_attend.hpp"
#include "status.hpp"

namespace {

using lce::aligned;
using lce::check_launch;
using lce::fail;
using lce::ok;
using lce::tuning;
using lce::kv4::kPage;

// Workgroups of 256 threads in a grid: threads are counted in 32 bits.
constexpr int64_t kMostGroups = (1LL << 24) - 1;

lce_status validate_cache(const lce_kv4_cache_desc *d) {
    if (!d) return fail(LCE_EINVAL, "desc is NULL");
    if (d->pages < 1 || d->kv_heads < 1)
        return fail(LCE_EINVAL, "pages %d and kv_heads %d must be >= 1", d->pages, d->kv_heads);
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
        return fail(LCE_EUNSUPPORTED, "head_dim %d is not 64, 128 or 256", d->head_dim);
    if (d->kv_heads > 65535)
        return fail(LCE_EUNSUPPORTED, "kv_heads %d exceeds 65535", d->kv_heads);
    return LCE_OK;
}

lce_status validate_tokens(const lce_kv4_cache_desc *d, int32_t type, int64_t tokens) {
    if (const lce_status st = validate_cache(d)) return st;
    if (type != LCE_FLOAT32 && type != LCE_FLOAT16 && type != LCE_BFLOAT16)
        return fail(LCE_EINVAL, "unknown type %d", type);
    if (tokens < 0 || tokens > INT32_MAX)
        return fail(LCE_EINVAL, "tokens %lld outside [0, 2^31)", (long long)tokens);
    // workgroups of at least 8 tokens of one head
    if ((tokens / 8 + 1) * d->kv_heads > kMostGroups)
        return fail(LCE_EUNSUPPORTED, "%lld tokens of %d heads: too many for one call",
                    (long long)tokens, d->kv_heads);
    return LCE_OK;
}

lce_status validate_query(const lce_kv4_cache_desc *d, const lce_kv4_query_desc *q) {
    if (const lce_status st = validate_cache(d)) return st;
    if (!q) return fail(LCE_EINVAL, "query is NULL");
    if (q->tokens < 0 || q->seqs < 1 || q->table_width < 1)
        return fail(LCE_EINVAL, "tokens %d must be >= 0, seqs %d and table_width %d >= 1",
                    q->tokens, q->seqs, q->table_width);
    if (q->q_heads < 1 || q->q_heads % d->kv_heads)
        return fail(LCE_EINVAL, "q_heads %d is not a multiple of kv_heads %d", q->q_heads,
                    d->kv_heads);
    if (q->table_width > 1 << 24)
        return fail(LCE_EUNSUPPORTED, "table_width %d: sequences of more than 2^30 tokens",
                    q->table_width);
    // rows and workgroups are counted in 32 bits
    if (((int64_t)q->tokens + q->seqs) * q->q_heads > INT32_MAX)
        return fail(LCE_EUNSUPPORTED, "%d tokens of %d heads in %d sequences: too many for one call",
                    q->tokens, q->q_heads, q->seqs);
    return LCE_OK;
}

lce_status validate_call(const lce_kv4_cache_desc *d, const lce_kv4_query_desc *q) {
    if (const lce_status st = validate_query(d, q)) return st;
    if (q->type != LCE_FLOAT16 && q->type != LCE_BFLOAT16)
        return fail(q->type == LCE_FLOAT32 ? LCE_EUNSUPPORTED : LCE_EINVAL,
                    "query type %d is not float16 or bfloat16", q->type);
    if (q->causal != 0 && q->causal != 1) return fail(LCE_EINVAL, "causal %d is not 0 or 1", q->causal);
    if (q->window < 0 || q->list < 0 || q->max_q < 0 || q->max_len < 0)
        return fail(LCE_EINVAL, "window %d, list %d, max_q %d and max_len %d must be >= 0",
                    q->window, q->list, q->max_q, q->max_len);
    // kernels count entries, and up to a workgroup's past the last, in 32 bits
    if (q->list > 1 << 24)
        return fail(LCE_EUNSUPPORTED, "list %d: more pages than a table has", q->list);
    return LCE_OK;
}

// What the workspace has room for: states of this many tiles of 16 rows, an eighth
// of it of 128.  More workgroups would not run at the same time anyway.
constexpr int64_t kMostParts = 4096;
static_assert(kMostParts / 2 <= lce::kv4::kTickets, "a ticket for each unit that is shared");

// Tiles of `rows` query rows of a cache head; with a list, of one token each.
int64_t tiles(const lce_kv4_cache_desc &d, const lce_kv4_query_desc &q, int rows, bool list) {
    const int64_t group = q.q_heads / d.kv_heads;
    return list ? q.tokens * ((group + rows - 1) / rows) : q.tokens * group / rows + q.seqs;
}

// Pages that a unit of work can have before it, as far as the call says.
int64_t most_pages(const lce_kv4_query_desc &q) {
    int64_t n = q.table_width;
    if (q.max_len > 0) n = std::min<int64_t>(n, (q.max_len + (int64_t)kPage - 1) / kPage);
    if (q.window > 0) n = std::min<int64_t>(n, ((int64_t)q.window + std::max(q.max_q, 1)) / kPage + 2);
    return n;
}

// The most rows that read the same pages, as far as the call says: the new tokens of
// a sequence (of a list: one), times the heads that share a cache head.
int64_t query_rows(const lce_kv4_cache_desc &d, const lce_kv4_query_desc &q) {
    const int64_t tokens = q.list ? 1 : q.max_q > 0 ? q.max_q : q.tokens / q.seqs;
    return tokens * (q.q_heads / d.kv_heads);
}

// Query rows of a tile of attention.  A tile takes a page's values out of 4 bits once
// for all its rows, but the more rows it has the fewer tiles there are, and fewer than
// run at a time (1024 of 32, 512 of 128) leave CUs without work; where no sequence is
// long, half as many tiles of 128 do.  Heads of 256 channels, and 32 rows of 128 in
// float16 (three pieces of a query, and more registers than there are), stay at 16.
// Measured in graphs over three caches (us, tiles of 16 / 32 / 128; 32 heads on 8 if not
// said otherwise):
//                                           bfloat16, 128     float16, 64   float16, 128
//   16 of 4064 tokens, 64 of them new        113 / 93 / 109   86 / 72 / 81  120 / - / 123
//   one of 5024, 1024 new                    118 / 98 / 118   91 / 81 / 87  131 / - / 132
//   one of 6048, 2048 new                   241 / 204 / 173 187 / 160 / 126 270 / - / 193
//   one of 8096, 4096 new                   515 / 425 / 362 393 / 334 / 258 565 / - / 404
//   four of up to 4512, up to 512 new         97 / 88 / 108   78 / 71 / 82  107 / - / 119
//   four of up to 5024, up to 1024 new      191 / 162 / 143 146 / 132 / 108 209 / - / 163
//   four of up to 6048, up to 2048 new      344 / 305 / 238 271 / 240 / 171 378 / - / 264
//   16 of up to 1024, up to 128 new           42 / 44 / 36    34 / 34 / 27   46 / - / 40
//   16 of up to 1024, up to 64, 64 heads      43 / 46 / 37    35 / 36 / 27   47 / - / 42
//   one prompt of 1024                        33 / 33 / 32    26 / 25 / 24   36 / - / 34
//   two of up to 5025, up to 359, 8 on 2      26 / 29 / 64    20 / 22 / 38   28 / - / 66
//   four prompts of up to 1943, 2 on 1        15 / 20 / 51    13 / 17 / 31   16 / - / 53
int tile_rows(const lce_kv4_cache_desc &d, const lce_kv4_query_desc &q) {
    if (d.head_dim > 128) return 16;
    const bool large = d.head_dim == 128 && q.type == LCE_FLOAT16;
    const int forced = tuning(LCE_TUNE_KV4_ROWS);
    if (q.list || forced == 16) return 16;
    if (forced == 128 || (forced == 32 && !large)) return forced;
    const int64_t most = query_rows(d, q), all = (int64_t)q.tokens * q.q_heads;
    const bool brief = most_pages(q) <= 16;
    if (most >= 128 && all >= 128 * (brief ? 256 : 512)) return 128;
    return most >= 256 && !large && all >= 32 * 1024 ? 32 : 16;
}

// Most states of one tile, of `units` tiles with room for `parts` states.
int64_t most_splits(int64_t units, int64_t parts) {
    return std::min<int64_t>(std::max<int64_t>(parts / std::max<int64_t>(units, 1), 1),
                             lce::kv4::kMostSplits);
}

// What states of attention take: with each height of a tile, up to a table's pages of
// them for each (a list splits no further), or as many as there is room for.  More
// tokens never take less, so that a workspace serves calls with fewer, too.
int64_t state_bytes(const lce_kv4_cache_desc &d, const lce_kv4_query_desc &q) {
    const int64_t splits = std::min<int64_t>(q.table_width, lce::kv4::kMostSplits);
    if (splits < 2) return 0;
    int64_t most = 0;
    for (const int rows : {16, 32, 128}) {
        if (rows > 16 && d.head_dim > 128) break;
        int64_t units = tiles(d, q, rows, false);
        if (rows == 16) units = std::max(units, tiles(d, q, rows, true));
        if (q.tokens == 0) units = 0;
        most = std::max(most, std::min(kMostParts * 16 / rows, units * d.kv_heads * splits) * rows);
    }
    return most * (d.head_dim + 4) * 4;
}

// What ranks of selection take.
int64_t rank_bytes(const lce_kv4_cache_desc &d, const lce_kv4_query_desc &q) {
    return (int64_t)q.tokens * d.kv_heads * q.table_width * 2;
}

struct Split {
    int chunk;    // pages per workgroup
    int splits;   // workgroups that share a unit, at most
};

// `pages` pages of each of `likely` units of work (the grid has room for `units`),
// `step` microseconds for a wave to take one: how many workgroups (of four waves)
// share a unit.  Sharing costs about `fixed` microseconds for the partial states,
// the ticket and the joining, and 0.06 for each state joined, so a unit is divided
// only where its pages take longer, and no further than `most` workgroups in all and
// `parts` states in the workspace.  `each`: the number of pages that a workgroup takes
// is a multiple of it, so that all waves are busy to the end.
Split split_pages(int64_t units, int64_t likely, int64_t pages, double step, double fixed,
                  int64_t most, int64_t parts, int64_t each) {
    const int64_t some = std::max<int64_t>(likely, 1);
    const int64_t room = most_splits(units, parts);
    int64_t chunk = std::max<int64_t>(pages, 1);
    if (const int t = tuning(LCE_TUNE_KV4_CHUNK)) {
        chunk = std::max(std::clamp<int64_t>(t, 1, chunk), (pages + room - 1) / room);
    } else {
        const double whole = pages * step / 4;
        // the least of whole / z + fixed + 0.06 z
        const double z = std::min(std::min((double)room, (double)most / some),
                                  std::sqrt(whole / 0.06));
        if (z > 1 && whole / z + fixed + 0.06 * z < whole)
            chunk = ((int64_t)std::ceil(pages / z) + each - 1) / each * each;
    }
    Split s;
    s.chunk = (int)chunk;
    s.splits = (int)std::max<int64_t>((pages + chunk - 1) / chunk, 1);
    return s;
}

void fill_query(lce::kv4::QueryParams &p, const lce_kv4_cache_desc &d, const void *cache,
                const lce_kv4_query_desc &q, const void *qp, const int32_t *table,
                const int32_t *q_start, const int32_t *lengths, const Split &s, void *workspace) {
    p.cache = static_cast<const uint8_t *>(cache);
    p.q = qp;
    p.table = table, p.q_start = q_start, p.lengths = lengths;
    p.q_token = q.q_token_stride, p.q_head = q.q_head_stride;
    p.pages = d.pages, p.kv_heads = d.kv_heads, p.group = q.q_heads / d.kv_heads;
    p.tokens = q.tokens, p.seqs = q.seqs, p.width = q.table_width;
    p.causal = q.causal, p.window = q.window, p.list = q.list;
    p.chunk = s.chunk;
    p.tickets = static_cast<int32_t *>(workspace);
}

}  // namespace

extern "C" {

lce_status lce_kv4_cache_size(const lce_kv4_cache_desc *desc, int64_t *bytes) {
    if (!bytes) return fail(LCE_EINVAL, "bytes output pointer is NULL");
    if (const lce_status st = validate_cache(desc)) return st;
    *bytes = (int64_t)desc->pages * desc->kv_heads * 76 * desc->head_dim;
    return ok();
}

lce_status lce_kv4_append(const lce_kv4_cache_desc *desc, void *cache, int32_t type,
                          const void *k, int64_t k_token_stride, int64_t k_head_stride,
                          const void *v, int64_t v_token_stride, int64_t v_head_stride,
                          const int64_t *slots, int64_t tokens, hipStream_t stream) {
    if (const lce_status st = validate_tokens(desc, type, tokens)) return st;
    if (tokens == 0) return ok();
    if (!cache || !k || !v || !slots) return fail(LCE_EINVAL, "cache/k/v/slots is NULL");
    if (!aligned(cache, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8))
        return fail(LCE_EALIGN, "cache, k and v must be 16-byte aligned, slots 8-byte");
    const int64_t unit = type == LCE_FLOAT32 ? 4 : 8;
    if (k_token_stride % unit || k_head_stride % unit || v_token_stride % unit ||
        v_head_stride % unit)
        return fail(LCE_EALIGN, "strides must be multiples of 16 bytes (%lld elements)",
                    (long long)unit);
    lce::kv4::AppendParams p;
    p.cache = static_cast<uint8_t *>(cache);
    p.k = k, p.v = v, p.slots = slots, p.tokens = tokens;
    p.k_token = k_token_stride, p.k_head = k_head_stride;
    p.v_token = v_token_stride, p.v_head = v_head_stride;
    p.pages = desc->pages, p.kv_heads = desc->kv_heads;
    lce::kv4::launch_append(p, type, desc->head_dim, stream);
    return check_launch("lce_kv4_append launch");
}

lce_status lce_kv4_read(const lce_kv4_cache_desc *desc, const void *cache, const int64_t *slots,
                        int64_t tokens, int32_t type, void *k, void *v, hipStream_t stream) {
    if (const lce_status st = validate_tokens(desc, type, tokens)) return st;
    if (tokens == 0) return ok();
    if (!cache || !k || !v || !slots) return fail(LCE_EINVAL, "cache/k/v/slots is NULL");
    if (!aligned(cache, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8))
        return fail(LCE_EALIGN, "cache, k and v must be 16-byte aligned, slots 8-byte");
    lce::kv4::ReadParams p;
    p.cache = static_cast<const uint8_t *>(cache);
    p.slots = slots, p.k = k, p.v = v, p.tokens = tokens;
    p.pages = desc->pages, p.kv_heads = desc->kv_heads;
    lce::kv4::launch_read(p, type, desc->head_dim, stream);
    return check_launch("lce_kv4_read launch");
}

lce_status lce_kv4_attention_workspace_size(const lce_kv4_cache_desc *desc,
                                            const lce_kv4_query_desc *query, int64_t *bytes) {
    if (!bytes) return fail(LCE_EINVAL, "bytes output pointer is NULL");
    if (const lce_status st = validate_query(desc, query)) return st;
    *bytes = LCE_KV4_WORKSPACE_ZERO + state_bytes(*desc, *query);
    return ok();
}

lce_status lce_kv4_select_workspace_size(const lce_kv4_cache_desc *desc,
                                         const lce_kv4_query_desc *query, int64_t *bytes) {
    if (!bytes) return fail(LCE_EINVAL, "bytes output pointer is NULL");
    if (const lce_status st = validate_query(desc, query)) return st;
    *bytes = LCE_KV4_WORKSPACE_ZERO + rank_bytes(*desc, *query);
    return ok();
}

lce_status lce_kv4_workspace_size(const lce_kv4_cache_desc *desc, const lce_kv4_query_desc *query,
                                  int64_t *bytes) {
    if (!bytes) return fail(LCE_EINVAL, "bytes output pointer is NULL");
    if (const lce_status st = validate_query(desc, query)) return st;
    *bytes = LCE_KV4_WORKSPACE_ZERO +
             std::max(state_bytes(*desc, *query), rank_bytes(*desc, *query));
    return ok();
}

lce_status lce_kv4_attention(const lce_kv4_cache_desc *desc, const void *cache,
                             const lce_kv4_query_desc *query, const void *q, const int32_t *table,
                             const int32_t *q_start, const int32_t *lengths, const int32_t *pages,
                             void *out, float *lse, void *workspace, int64_t workspace_bytes,
                             hipStream_t stream) {
    if (const lce_status st = validate_call(desc, query)) return st;
    const float scale_log2 = query->scale * 1.44269504088896341f;
    if (!(query->scale > 0.0f) || !std::isfinite(scale_log2))
        return fail(LCE_EINVAL, "scale %g is not a finite number > 0", query->scale);
    if (query->tokens == 0) return ok();
    if (!cache || !q || !table || !q_start || !lengths || !out || !workspace)
        return fail(LCE_EINVAL, "cache/q/table/q_start/lengths/out/workspace is NULL");
    if (query->list > 0 && !pages) return fail(LCE_EINVAL, "list %d needs pages", query->list);
    if (!aligned(cache, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16))
        return fail(LCE_EALIGN, "cache, q, out and workspace must be 16-byte aligned");
    if (!aligned(table, 4) || !aligned(q_start, 4) || !aligned(lengths, 4) || !aligned(pages, 4) ||
        !aligned(lse, 4))
        return fail(LCE_EALIGN, "table, q_start, lengths, pages and lse must be 4-byte aligned");
    if (query->q_token_stride % 8 || query->q_head_stride % 8)
        return fail(LCE_EALIGN, "q strides must be multiples of 8 elements");
    int64_t need = 0;
    if (const lce_status st = lce_kv4_attention_workspace_size(desc, query, &need)) return st;
    if (workspace_bytes < need)
        return fail(LCE_EINVAL, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                    (long long)need);

    const bool list = query->list > 0;
    const int rows = tile_rows(*desc, *query);
    const int64_t units = tiles(*desc, *query, rows, list) * desc->kv_heads;
    const double size = desc->head_dim / 128.0;
    const int64_t slots = desc->head_dim > 128 ? 512 : 768;   // workgroups that run at a time
    // Lists are of one length: half of the workgroups that run at a time, each with more
    // pages to hide latencies behind; windows mostly: all of them.  Sequences are of
    // different lengths, of which the call knows the longest: if they were all as long,
    // 7/4 of what runs at a time, which is about all of it when they are not.  Where a
    // sequence has several tiles already, 512, and states of all their rows to store and
    // join.  Measured in graphs over three caches (us; up to so many tokens, new ones,
    // heads; 128 channels, one new token and 32 heads on 8 if not said otherwise; the last
    // of 64 channels):
    //   pages a workgroup        choice     8    12    16    24    32    48    64   all
    //   1 of 20001                 13.3  15.0  13.3  13.6  14.4  16.1  19.8  23.6  83.0
    //   32 of up to 8192           33.2  41.0  40.0  38.1  37.3  33.7  35.2  35.8  48.4
    //   4 of up to 65536           46.9  53.5  52.3  47.1  47.9  41.2  45.9  49.9   308
    //   64 of 8192, 64 heads       54.1  60.2  59.5  60.6  60.3  59.1  55.7  57.3  55.9
    //   48 of 12000, 64 heads      62.5  70.3  70.6  70.2  70.2  68.5  69.2  64.4  75.4
    //   128 lists of 64            17.5  21.5  18.3  17.3  17.4  18.7  22.3  25.1  24.6
    //   120 lists of 24, of 256    19.3  21.7  19.3  21.0  21.1  21.1  21.2  21.1  21.0
    //   2 of 5025, 359, 8 on 2     25.1  38.4  31.6  30.9  25.8  26.1  25.1  26.5  24.9
    //   16 of 4096, 5, 24 on 4     13.2  13.5  12.5  12.7  13.6  15.3  18.3  20.3  20.3
    const int64_t seen = most_pages(*query);
    const int64_t most = list ? std::min<int64_t>(query->list, seen) : seen;
    const int64_t each = query_rows(*desc, *query);
    const bool several = !list && each > 64;
    // the grid has a tile to spare for each sequence; most calls have fewer (counted in
    // floating point: max_q is the caller's word)
    const double spread = (list ? query->tokens : query->seqs) * (double)desc->kv_heads;
    const int64_t likely = (int64_t)std::min((double)units, spread * ((each + rows - 1) / rows));
    const Split s =
        rows == 128
            ? split_pages(units, likely, most, 2 + 2 * size, 4 + 8 * size, 512, kMostParts / 8, 1)
            : split_pages(units, likely, most, 0.4 + 0.4 * size,
                          (0.5 + 1.3 * size) * (several ? 2.5 : 1.0),
                          list ? slots / 2 : query->window ? slots : several ? 512 : 7 * slots / 4,
                          kMostParts * 16 / rows, 4);
    // Loads past the caches where no other tile reads the same pages, heads have 128
    // channels (of others lines are read in two halves) and the whole is long enough.  The
    // bounds are of what the call could read, all sequences as long as the longest: of
    // those below, they read half of it or less.  Measured in graphs (us, through the
    // caches / past them; one token each of n sequences of up to ..., or n lists):
    //   could read  read, MB
    //      143         72   16 of 8192, 64 heads on 8       21.9 / 23.9
    //      214        106   24 of 8192, 64 on 8             31.1 / 31.2
    //      231        106   32 of 53109, 16 on 1            46.4 / 45.7
    //      250        118   28 of 8192, 64 on 8             32.6 / 31.6
    //      285        132   32 of 8192, 64 on 8             36.4 / 34.0
    //      285        100   128 of 2000, 64 on 8            30.4 / 30.6
    //      349        175   16 of 20000, 32 on 8            52.6 / 49.4
    //      570        238   64 of 8192, 64 on 8             58.4 / 53.4
    //       71         61   16 lists of 64 pages            17.1 / 18.4
    //      107         95   24 lists of 64                  24.2 / 24.6
    //      134        135   60 lists of 32                  29.5 / 27.2
    //      214        192   48 lists of 64                  43.7 / 39.0
    const bool once = each <= 16 && 68.0 * desc->head_dim * most * likely >=
                                        (list ? 120 << 20 : 240 << 20);
    lce::kv4::AttendParams p;
    fill_query(p, *desc, cache, *query, q, table, q_start, lengths, s, workspace);
    p.named = list ? pages : nullptr;
    p.out = out;
    p.lse = lse;
    p.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + LCE_KV4_WORKSPACE_ZERO);
    p.scale_log2 = scale_log2;
    p.turn = units % 8 == 0 && desc->kv_heads % 8 ? (int)units : 0;
    if (units > kMostGroups)
        return fail(LCE_EUNSUPPORTED, "%lld tiles: too many for one call", (long long)units);
    const dim3 grid((unsigned)units, (unsigned)s.splits);
    static const char *const kNames[2][4] = {
        {"kv4-list", "kv4-16", "kv4-32", "kv4-128"},
        {"kv4-list-split", "kv4-16-split", "kv4-32-split", "kv4-128-split"}};
    lce::g_last_schedule = kNames[s.splits > 1][list ? 0 : rows == 16 ? 1 : rows == 32 ? 2 : 3];
    if (rows == 128)
        lce::kv4::launch_attend128(p, query->type, desc->head_dim, grid, stream);
    else
        lce::kv4::launch_attend16(p, query->type, desc->head_dim, rows, once, grid, stream);
    return check_launch("lce_kv4_attention launch");
}

lce_status lce_kv4_select(const lce_kv4_cache_desc *desc, const void *cache,
                          const lce_kv4_query_desc *query, const void *q, const int32_t *table,
                          const int32_t *q_start, const int32_t *lengths, int32_t keep_first,
                          int32_t keep_last, int32_t *pages, void *workspace,
                          int64_t workspace_bytes, hipStream_t stream) {
    if (const lce_status st = validate_call(desc, query)) return st;
    if (query->list < 1 || keep_first < 0 || keep_last < 0)
        return fail(LCE_EINVAL, "list %d must be >= 1, keep_first %d and keep_last %d >= 0",
                    query->list, keep_first, keep_last);
    if ((int64_t)query->q_heads / desc->kv_heads * desc->head_dim > 65280)
        return fail(LCE_EUNSUPPORTED, "%d query heads of %d channels a cache head: past 65280",
                    query->q_heads / desc->kv_heads, desc->head_dim);
    if (query->tokens == 0) return ok();
    if (!cache || !q || !table || !q_start || !lengths || !pages || !workspace)
        return fail(LCE_EINVAL, "cache/q/table/q_start/lengths/pages/workspace is NULL");
    if (!aligned(cache, 16) || !aligned(q, 16) || !aligned(workspace, 16))
        return fail(LCE_EALIGN, "cache, q and workspace must be 16-byte aligned");
    if (!aligned(table, 4) || !aligned(q_start, 4) || !aligned(lengths, 4) || !aligned(pages, 4))
        return fail(LCE_EALIGN, "table, q_start, lengths and pages must be 4-byte aligned");
    if (query->q_token_stride % 8 || query->q_head_stride % 8)
        return fail(LCE_EALIGN, "q strides must be multiples of 8 elements");
    int64_t need = 0;
    if (const lce_status st = lce_kv4_select_workspace_size(desc, query, &need)) return st;
    if (workspace_bytes < need)
        return fail(LCE_EINVAL, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                    (long long)need);

    const int64_t units = (int64_t)query->tokens * desc->kv_heads;
    if (units > kMostGroups)
        return fail(LCE_EUNSUPPORTED, "%lld tokens and heads: too many for one call",
                    (long long)units);
    // a window hides pages but does not renumber them: all up to the last count
    lce_kv4_query_desc all = *query;
    all.window = 0;
    // Measured in graphs (us by pages a workgroup, one token of each sequence, heads of 128
    // if not said otherwise; * is the choice):
    //                                         8     16     32     64    128    all
    //   1 of 20001, 32 heads on 8            8.6*   8.7    8.9   10.0   12.5   19.1
    //   1 of 100000, 32 on 8                15.1*  15.1   14.5   15.0   17.4   33.3
    //   8 of up to 8192, 32 on 8             8.1*   8.2    8.2    9.4   10.8   10.8
    //   32 of up to 2048, 32 on 8            7.2    7.3    6.2*   6.2    6.2    6.2
    //   60 of up to 3000, 16 on 1 of 256     8.9*   8.9    9.8    9.9    9.8   10.0
    //   64 of up to 8192, 64 on 8           17.5   17.6   15.5*  15.4   15.4   15.4
    //   4 of up to 65536, 32 on 2           12.9*  12.7   12.5   14.3   17.2   35.7
    //   32 of up to 32768, 64 on 8          22.6   22.6   22.6   23.5*  23.8   30.7
    //   128 of up to 16384, 64 on 8         31.2   31.3   31.4   31.3   33.7*  33.0
    const Split s = split_pages(units, units, most_pages(all), 0.5, 3.5, 2048, kMostParts, 1);
    lce::kv4::SelectParams p;
    fill_query(p, *desc, cache, *query, q, table, q_start, lengths, s, workspace);
    p.keep_first = keep_first, p.keep_last = keep_last;
    p.chosen = pages;
    p.ranks = reinterpret_cast<uint16_t *>(static_cast<char *>(workspace) + LCE_KV4_WORKSPACE_ZERO);
    lce::kv4::launch_select(p, query->type, desc->head_dim,
                            dim3((unsigned)units, (unsigned)s.splits), stream);
    return check_launch("lce_kv4_select launch");
}

}  // extern "C"
