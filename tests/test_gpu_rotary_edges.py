"""Rotary positions on the GPU at the ends of what their entry point takes."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from tests import kv8_util as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("base", [10000.0, 500000.0])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_of_ordinary_frequencies(base, interleaved):
    """Against angles whose frequencies are not rounded: each is held to half of 2^-64 turns and
    what the 64-bit quotient leaves (a tenth of that), the angle to 2^-33 turns, products and
    series to 2^-21 of the pair's size."""
    plan = lce.Rotary(64, base=base, interleaved=interleaved)
    at = [0, 1, -1, 2 ** 20 + 1, 2 ** 31 - 1, -2 ** 31, 2 ** 32 + 5, 2 ** 36 + 3, -2 ** 40 - 7, 2 ** 45 + 9,
          2 ** 52 + 1]
    x = np.random.default_rng(1).standard_normal((len(at), 3, 64)).astype(np.float32)
    turns = [Fraction(f) / (2 * ref.PI) for f in plan.freqs.tolist()]
    angles = np.array([[2 * np.pi * float(p * t % 1) for t in turns] for p in at])
    want = ref.rotary(x, angles, plan.freqs.numpy(), 1.0, interleaved)
    got = lce.rotary(plan, torch.tensor(at).cuda(), torch.from_numpy(x).cuda()).cpu().double().numpy()
    pair = (slice(0, 64, 2), slice(1, 64, 2)) if interleaved else (slice(0, 32), slice(32, 64))
    size = np.hypot(x[..., pair[0]], x[..., pair[1]]).astype(np.float64)
    far = 2 * np.pi * 0.6 * 2.0 ** -64 * np.abs(np.array(at, np.float64))[:, None, None]
    for part in pair:
        bound = (2.0 ** -21 + far) * size + 2.0 ** -24 * np.abs(want[..., part])
        off = np.abs(got[..., part] - want[..., part]) - bound
        assert off.max() <= 0, (off.max(), np.argwhere(off > 0)[:4].tolist())
