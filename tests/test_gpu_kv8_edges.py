"""Attention over the 8-bit cache at the ends of what its entry point takes: the smallest
scales, queries that are not finite, calls that the smaller tests do not reach."""
import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
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
