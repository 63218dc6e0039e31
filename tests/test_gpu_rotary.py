"""Rotary positions on the GPU against complex numbers in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from tests import kv8_util as ref

pytestmark = pytest.mark.gpu


def tensors(seed, n, heads, dim, dtype):
    rng = np.random.default_rng(seed)
    return [torch.from_numpy(rng.standard_normal((n, h, dim))).to(ref.DTYPES[dtype]) for h in heads]


def check(plan, at, xs, got, dtype, backward=False):
    """Angles are off by at most 2^-33 turns and half a last place of an eighth turn's
    float32 (2^-25), the series and their products by a few last places: 2^-21 of the
    pair's size in all; the result by half a last place of its type."""
    for x, y in zip(xs, got):
        x = x.double().numpy()
        want = ref.rotary(x, at, plan.freqs.numpy(), plan.scale, plan.interleaved, backward)
        r = plan.rot_dim
        size = np.zeros_like(x)
        a, b = ((slice(0, r, 2), slice(1, r, 2)) if plan.interleaved
                else (slice(0, r // 2), slice(r // 2, r)))
        size[..., a] = size[..., b] = np.hypot(x[..., a], x[..., b]) * abs(plan.scale)
        bound = 2.0 ** -21 * size + ref.HALF_ULP[dtype] * 1.01 * np.abs(want)
        if dtype == "f16":
            bound += 2.0 ** -25
        bound[..., r:] = 0
        off = np.abs(y.cpu().double().numpy() - want) - bound
        assert off.max() <= 0, (off.max(), np.argwhere(off > 0)[:4].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (64, 64), (256, 64), (128, 32), (80, 80), (96, 48),
                                     (80, 20), (64, 2), (6, 4), (2, 2), (7, 6), (72, 32)])
def test_layouts(dim, rot, interleaved, dtype):
    plan = lce.Rotary(dim, rot_dim=rot, interleaved=interleaved)
    at = np.array([0, 1, 2, 3, 1000, 4095, 131071, 10 ** 6 + 3, 5, 17, 63])
    for heads in ((5, 1), (3,)):
        xs = tensors(dim, len(at), heads, dim, dtype)
        for backward in (False, True):
            got = lce.rotary(plan, torch.from_numpy(at).cuda(), *(x.cuda() for x in xs),
                             backward=backward)
            check(plan, at, xs, got if len(heads) == 2 else (got,), dtype, backward)


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
                                     dict(scaling="yarn", factor=16.0, original=4096),
                                     dict(scaling="yarn", factor=2.0, original=100), dict(base=500000.0),
                                     dict(freqs=np.linspace(-7, 7, 64)), dict(scale=-0.25)], ids=str)
def test_frequencies(scaling):
    plan = lce.Rotary(128, **scaling)
    at = np.arange(0, 300000, 997)
    xs = tensors(1, len(at), (4, 2), 128, "f32")
    check(plan, at, xs, lce.rotary(plan, torch.from_numpy(at).cuda(), *(x.cuda() for x in xs)), "f32")


def test_far_and_negative_positions():
    """Turns at any position, against whole numbers (float64 does not hold these angles)."""
    freqs = 2 * np.pi * 2.0 ** -np.arange(3, 19)
    plan = lce.Rotary(32, freqs=freqs)
    at = np.array([2 ** 62 + 12345, -(2 ** 63), -1, -77777, 2 ** 40 + 1, 2 ** 63 - 1, 2 ** 31, -2 ** 31])
    xs = tensors(2, len(at), (3, 1), 32, "f32")
    check(plan, ref.far_angles(at, freqs), xs, lce.rotary(plan, torch.from_numpy(at).cuda(), *(x.cuda() for x in xs)), "f32")


def test_long_calls_share_angles():
    """More heads a thread than one, and more tokens than a grid's first groups."""
    for dtype, n, heads in (("bf16", 3000, (33, 7)), ("f32", 1500, (32, 32)), ("f16", 9000, (8, 8))):
        plan = lce.Rotary(128, rot_dim=64)
        at = np.random.default_rng(3).integers(0, 100000, n)
        xs = tensors(4, n, heads, 128, dtype)
        check(plan, at, xs, lce.rotary(plan, torch.from_numpy(at).cuda(), *(x.cuda() for x in xs)), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", [128, 48])
def test_views_and_in_place(dtype, rot):
    plan = lce.Rotary(128, rot_dim=rot)
    at = torch.arange(37).cuda()
    rows = tensors(5, 37, (9,), 128, dtype)[0].cuda()
    q, k = rows[:, :5], rows[:, 5:7]
    want = lce.rotary(plan, at, q.contiguous(), k.contiguous())
    assert all(torch.equal(a, b) for a, b in zip(want, lce.rotary(plan, at, q, k)))
    first = q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(want[0], lce.rotary(plan, at, first))
    keep = rows.clone()
    got = lce.rotary(plan, at, q, k, out=(q, k))
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(rows[:, 7:], keep[:, 7:])
    # one in place, one not; and addresses that 16-byte loads do not fit
    odd = torch.zeros(37, 5, 129, dtype=rows.dtype, device="cuda")[..., 1:]
    odd.copy_(keep[:, :5])
    out = torch.empty_like(want[1])
    lce.rotary(plan, at, odd, keep[:, 5:7], out=(odd, out))
    assert torch.equal(odd, want[0]) and torch.equal(out, want[1])


def test_gradients():
    """backward is the transpose of the turn, and agrees with differences."""
    plan = lce.Rotary(64, rot_dim=48, interleaved=True, scaling="yarn", factor=8.0)
    at = torch.arange(100, 2000, 61).cuda()
    x, y = (t.cuda() for t in tensors(6, len(at), (3, 3), 64, "f32"))
    a = (lce.rotary(plan, at, x).double() * y.double()).sum()
    b = (x.double() * lce.rotary(plan, at, y, backward=True).double()).sum()
    # sums of 64 * 3 * 32 products, each off by 2^-21
    assert abs(a - b) <= 2.0 ** -21 * plan.scale * (x.double().norm() * y.double().norm())
    grad = lce.rotary(plan, at, y, backward=True)
    # the turn is linear: a central difference of step 1 is exact but for rounding
    for i, j, c in ((0, 0, 0), (5, 1, 47), (31, 2, 48), (17, 0, 63), (3, 2, 16)):
        d = torch.zeros_like(x)
        d[i, j, c] = 1
        up, down = (lce.rotary(plan, at, x + s * d).double() for s in (1, -1))
        diff = float(((up - down) / 2 * y.double()).sum())
        size = float(y[i, j].double().abs().sum() * (x[i, j].double().abs().max() + 1)) * plan.scale
        assert abs(diff - float(grad[i, j, c])) <= 2.0 ** -20 * size


def test_graph_and_streams():
    plan = lce.Rotary(128)
    at = torch.arange(7).cuda()
    q, k = (t.cuda() for t in tensors(7, 7, (4, 2), 128, "bf16"))
    lce.rotary(plan, at, q, k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lce.rotary(plan, at, q, k)
    for i in range(4):
        at += 1000 * i
        q.mul_(0.5)
        graph.replay()
        want = lce.rotary(plan, at, q, k)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_empty_and_untouched():
    plan = lce.Rotary(64)
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16).cuda()
    assert lce.rotary(plan, torch.empty(0, dtype=torch.int64).cuda(), none).shape == (0, 4, 64)
