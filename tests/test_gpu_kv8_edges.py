"""Attention over the 8-bit cache at the ends of what its entry point takes: the smallest
scales, queries that are not finite, calls that the smaller tests do not reach."""
import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from tests import kv8_exact as exact
from tests import kv8_util as ref

pytestmark = pytest.mark.gpu


def check(batch, scale=None, weights=None, **kw):
    """The call against the oracle, within the bounds that the oracle derives."""
    opts = {k: v for k, v in kw.items() if k in ("causal", "window", "cap", "slopes", "prefix")}
    scale = batch.dim ** -0.5 if scale is None else float(np.float32(scale))
    want, want_lse, bound, lse_bound = batch.attention(scale, weights=weights, **opts)
    opts["softcap"] = opts.pop("cap", 0.0)
    for name, dtype in (("slopes", torch.float32), ("prefix", torch.int32)):
        if opts.get(name) is not None:
            opts[name] = torch.as_tensor(opts[name], dtype=dtype).cuda()
    out, lse = lce.kv8_attention(*batch.device(lce), scale=scale, return_lse=True, **opts)
    got, got_lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    assert np.isfinite(got).all(), np.argwhere(~np.isfinite(got))[:5].tolist()
    off = np.abs(got - want) - bound
    assert off.max() <= 0, (off.max(), np.argwhere(off > 0)[:5].tolist())
    seen = np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(got_lse), ~seen)
    assert (np.abs(got_lse - want_lse)[seen] <= lse_bound[seen]).all()
    return out, lse


@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,scale", [("f16", 1e-6), ("f16", 1e-9), ("bf16", 1e-9), ("bf16", 1e-38)])
@pytest.mark.parametrize("zero", [False, True])
def test_smallest_scales(dim, dtype, scale, rows, zero):
    """Scales that leave next to nothing of a score, where a step has tokens that some row does
    not see: all that it sees weigh the same, and what is hidden nothing.  Half a page that no
    row sees, a window that begins in a page's second half, and keys of zero have the smallest
    block scale."""
    every = slice(None)
    odd = [(b, every, every, every, "k", 0.0) for b in range(3)] if zero else []
    batch = ref.Batch(dim + rows, [10, 70, 130], [3, 40, 2], 4, 2, dim, dtype, odd=odd)
    with lce.tuning(kv8_rows=rows):
        for opts in (dict(), dict(window=20), dict(causal=False)):
            check(batch, scale, **opts)


@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("opts", [dict(), dict(softcap=5.0), dict(softcap=1e6), dict(slopes=True),
                                  dict(softcap=5.0, slopes=True)], ids=str)
def test_an_infinity_in_a_query_makes_its_row_nan(dim, dtype, rows, opts):
    """Also where its products with the keys all are the same infinity, which no score of the
    row is larger than, or which a cap makes finite; rows beside it stay, and a row that sees
    nothing is 0."""
    every = slice(None)
    odd = [(b, every, every, 7, "k", -1.0) for b in range(3)]
    batch = ref.Batch(dim + rows, [1, 70, 2], [1, 40, 3], 4, 2, dim, dtype, odd=odd)
    inf = float("inf")
    batch.q[0, 0, 7], batch.q[3, 2, 7], batch.q[20, 1, 7], batch.q[33, 3, 7] = inf, inf, -inf, -inf
    batch.q[41, 0, 7] = inf                        # before the sequence's beginning
    batch.q[42, 3, 7] = inf
    if opts.get("slopes"):
        opts = dict(opts, slopes=torch.tensor([0.5, 0.0, 0.1, 0.25]).cuda())
    cache, q, table, start, lengths = batch.device(lce)
    with lce.tuning(kv8_rows=rows):
        out, lse = lce.kv8_attention(cache, q, table, start, lengths, return_lse=True, **opts)
        clean = torch.where(torch.isinf(q), 0.0, q)
        want, want_lse = lce.kv8_attention(cache, clean, table, start, lengths, return_lse=True,
                                           **opts)
    bad = torch.zeros(44, 4, dtype=torch.bool, device="cuda")
    for token, head in ((0, 0), (3, 2), (20, 1), (33, 3), (42, 3)):
        bad[token, head] = True
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.equal(out[~bad], want[~bad]) and torch.equal(lse[~bad], want_lse[~bad])
    assert not out[41].any() and torch.isneginf(lse[41]).all()


SLOPES = [0.5, 0.0, -0.01, 2.0, 0.1, 1.0, 0.01, 0.3]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("opts", [
    dict(slopes=SLOPES), dict(slopes=SLOPES, causal=False), dict(slopes=SLOPES, window=90),
    dict(cap=5.0, slopes=SLOPES), dict(cap=1e6), dict(cap=1e6, slopes=SLOPES, causal=False),
    dict(cap=5.0, slopes=SLOPES, prefix=[600, 2, 0, 70, 310])], ids=str)
def test_every_change_of_scores_in_every_tile(dim, dtype, rows, opts):
    """Biases by distance, far caps and both in tiles of each height and in calls of many rows,
    over several pages, whole and split."""
    batch = ref.Batch(dim + rows, [700, 130, 1, 64, 333], [40, 9, 1, 2, 33], 8, 2, dim, dtype, loud=3.0)
    want = batch.attention(dim ** -0.5, **opts)
    batch.attention = lambda *args, **kw: want     # the same for every split
    for chunk in (0, 1, 3):
        with lce.tuning(kv8_rows=rows, kv8_chunk=chunk):
            check(batch, **opts)
            name = lce.last_schedule()
        assert name.startswith("kv8-16" if dim == 256 else f"kv8-{rows}")
        assert chunk != 1 or name.endswith("-split")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("opts", [dict(), dict(cap=20.0), dict(slopes=SLOPES[:4]),
                                  dict(cap=20.0, slopes=SLOPES[:4], window=200)], ids=str)
def test_pages_that_go_past_the_caches(dim, dtype, opts):
    """Calls whose table says that they read more than 240 MiB, of single tokens and of a few,
    load pages past the caches; the same calls with a table as wide as their pages do not, and
    give the same bits where they split the work alike."""
    lengths = [0, 1, 15, 64, 130, 3000, 300, 65]
    queries = [0, 1, 2, 1, 3, 1, 2, 1]
    seqs, width = len(lengths), 20000
    assert 128 * dim * width * seqs >= 240 << 20
    batch = ref.Batch(dim, lengths, queries, 4, 2, dim, dtype, width=width)
    out, lse = check(batch, **opts)
    kw = dict(softcap=opts.get("cap", 0.0), window=opts.get("window", 0), return_lse=True)
    if "slopes" in opts:
        kw["slopes"] = torch.tensor(opts["slopes"]).cuda()
    cache, q, table, start, lens = batch.device(lce)
    # one workgroup a tile in both
    wide, narrow = table, table[:, :-(-max(lengths) // ref.PAGE)].contiguous()
    got = []
    for t in (wide, narrow):
        with lce.tuning(kv8_chunk=width // 2):
            got.append(lce.kv8_attention(cache, q, t, start, lens, **kw))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("dtype,weights", [("bf16", 2.0 ** -14), ("f16", 2.0 ** -20)])
@pytest.mark.parametrize("q_heads,kv_heads,dim", [(8, 2, 64), (7, 1, 128), (16, 2, 256)])
@pytest.mark.parametrize("chunk", [0, 1])
def test_weights_of_two_parts_where_results_are_small(q_heads, kv_heads, dim, dtype, weights, chunk):
    """Exact scores, and values that nearly cancel: a weight rounded once would show."""
    b = exact.batch(dim, [5, 30, 100], [1, 1, 1], q_heads, kv_heads, dim, dtype)
    want, bound, _ = exact.expected(b, weights)
    with lce.tuning(kv8_chunk=chunk):
        out = lce.kv8_attention(*b.device(lce), scale=exact.SCALE).cpu().double().numpy()
    off = np.abs(out - want) - bound
    assert off.max() <= 0, (off.max(), np.argwhere(off > 0)[:5].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_a_sequences_bits_do_not_depend_on_the_others(dtype, rows):
    """A sequence alone and beside others, of longer and shorter lengths, with the same hints
    and the same pages a workgroup."""
    lengths, queries = [900, 70, 300, 5, 450], [4, 1, 40, 5, 1]
    batch = ref.Batch(10, lengths, queries, 8, 2, 128, dtype)
    cache, q, table, start, lens = batch.device(lce)
    kw = dict(return_lse=True, max_q=40, max_len=900)
    with lce.tuning(kv8_rows=rows, kv8_chunk=3):
        out, lse = lce.kv8_attention(cache, q, table, start, lens, **kw)
        for b, n in enumerate(queries):
            at = slice(int(batch.start[b]), int(batch.start[b]) + n)
            one, one_lse = lce.kv8_attention(cache, q[at], table[b:b + 1],
                                             torch.tensor([0, n], dtype=torch.int32).cuda(),
                                             lens[b:b + 1], **kw)
            assert torch.equal(one, out[at]) and torch.equal(one_lse, lse[at]), b
