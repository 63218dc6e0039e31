"""Host side of the rotary positions, on the CPU: frequencies at the ends of what scalings take,
and refusals.  Nothing is ever launched; fake non-null pointers are plain integers."""
import ctypes
import math

import numpy as np
import pytest

import paper_2011_09398_amd as lce
from paper_2011_09398_amd import build as lce_build

P = 0x10000


@pytest.fixture(scope="module", autouse=True)
def built():
    if lce_build.is_stale():
        lce_build.build()


def yarn(rot, base, factor, original):
    out, scale = (ctypes.c_double * (rot // 2))(), ctypes.c_float()
    assert lce.lib().lce_rotary_frequencies(rot, base, lce.ROTARY_SCALING["yarn"], factor, original,
                                            out, ctypes.byref(scale)) == lce.LCE_OK
    return np.array(out[:])


@pytest.mark.parametrize("rot,base,original", [
    (32, 100.0, 1e7), (16, 10.0, 1e6), (64, 500.0, 1e8), (2, 2.0, 1e9), (2, 1e4, 1e5), (4, 1.5, 4096),
    (128, 1e4, 1e12), (128, 1e4, 4096), (64, 1e4, 100), (64, 5e5, 8192), (8, 1.001, 1e4)])
@pytest.mark.parametrize("factor", [1.0, 8.0])
def test_yarn_by_the_number_of_turns(rot, base, original, factor):
    """Pairs that turn more than 32 times over the original context keep their frequency, those
    that turn less than once are slowed by all of the factor, the others by some of it, and no
    pair by less than a faster one.  (The bounds are whole pairs: a pair's turns to the next
    one's are base^(2 / rot) to 1.)"""
    plain = base ** (-2.0 * np.arange(rot // 2) / rot)
    ratio = plain / yarn(rot, base, factor, original)
    turns, step = original * plain / (2 * math.pi), base ** (2.0 / rot)
    assert np.allclose(ratio[turns > 32 * step], 1, rtol=1e-13)
    assert np.allclose(ratio[turns * step < 1], factor, rtol=1e-13)
    assert (ratio >= 1 - 1e-13).all() and (ratio <= factor * (1 + 1e-13)).all()
    assert (np.diff(ratio) >= -1e-13).all()


def rows(**kw):
    return lce.RotaryRows(**{**dict(heads=4, x=P, y=P, x_token_stride=256, x_head_stride=64,
                                    y_token_stride=256, y_head_stride=64), **kw})


def call(q, k=None, **kw):
    d = lce.RotaryDesc(**{**dict(tokens=3, head_dim=64, rot_dim=64, type=2, interleaved=0, backward=0,
                                 scale=1.0), **kw})
    return lce.lib().lce_rotary(ctypes.byref(d), P, P, ctypes.byref(q),
                                ctypes.byref(k) if k is not None else None, None)


def test_queries_and_keys_in_one_place_are_refused():
    """Results of one where the other's are written or are still to be read."""
    far = 1 << 20
    for q, k in ((rows(y=far), rows(y=far)), (rows(), rows()), (rows(x=P, y=far), rows(x=far, y=P)),
                 (rows(y=far), rows(x=far, y=2 * far)), (rows(x=far, y=2 * far), rows(y=far))):
        assert call(q, k) == lce.LCE_EINVAL
        assert "q and k" in lce.last_error()


def test_counts_past_64_bits_are_refused():
    """Tokens times heads times channels that an int64 does not hold."""
    wide = dict(heads=1 << 20, y_head_stride=65536, y_token_stride=1 << 36)
    for x in (P, P + 2):                           # 16 bytes at a time, and one channel
        assert call(rows(x=x, y=1 << 30, **wide), tokens=2 ** 31 - 1, head_dim=65536,
                    rot_dim=65536) == lce.LCE_EUNSUPPORTED
    assert call(rows(x=P + 2, **{**wide, "heads": (1 << 20) - 1}), tokens=2 ** 30 + 12345,
                head_dim=65536, rot_dim=65534) == lce.LCE_EUNSUPPORTED
