"""Attention over the 8-bit cache at the ends of what its entry point takes: the smallest
scales, and calls that the smaller tests do not reach."""
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
