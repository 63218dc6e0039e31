"""What the GPU's test of two-part weights is able to see, on the CPU: weights rounded once are
outside its bounds, weights of two parts within."""
import numpy as np
import pytest
import torch

from tests import kv8_exact as exact
from tests import kv8_util as ref

# the bits that are left of a weight: see test_gpu_kv8_edges
CASES = [("bf16", 2.0 ** -14, 0xFFFF0000), ("f16", 2.0 ** -20, 0xFFFFE000)]


def rounded(x, dtype):
    return torch.from_numpy(np.asarray(x)).to(ref.DTYPES[dtype]).double().numpy()


@pytest.mark.parametrize("dtype,weights,mask", CASES)
@pytest.mark.parametrize("q_heads,kv_heads,dim", [(8, 2, 64), (7, 1, 128), (16, 2, 256)])
def test_weights_rounded_once_would_show(q_heads, kv_heads, dim, dtype, weights, mask):
    b = exact.batch(dim, [5, 30, 100], [1, 1, 1], q_heads, kv_heads, dim, dtype)
    want, bound, parts = exact.expected(b, weights)
    seen = {}
    for i, h, w, v in parts:
        w32 = w.astype(np.float32)
        high = (w32.view(np.uint32) & np.uint32(mask)).view(np.float32)
        low = ((w32 - high).view(np.uint32) & np.uint32(mask)).view(np.float32)
        once = rounded(w, dtype)
        two = high.astype(np.float64) + low.astype(np.float64)
        for name, got in (("two", two @ v / w.sum()), ("once", once @ v / w.sum()),
                          ("once, by their sum", once @ v / once.sum())):
            off = np.abs(rounded(got, dtype) - want[b.start[i], h]) - bound[b.start[i], h]
            seen[name] = seen.get(name, 0) + int((off > 0).sum())
    total = sum(v.shape[1] for _, _, _, v in parts)
    assert seen["two"] == 0
    assert seen["once"] > total // 4 and seen["once, by their sum"] > total // 4, (seen, total)
