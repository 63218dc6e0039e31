"""Host side of the 8-bit cache's and the rotary positions' entry points, on the CPU: sizes,
frequencies and refusals.  Nothing is ever launched; fake non-null pointers are plain
integers."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from paper_2011_09398_amd import build as lce_build
from tests import kv8_util as ref

P = 0x10000
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def built():
    if lce_build.is_stale():
        lce_build.build()


def cache(**kw):
    return lce.KV8CacheDesc(**{**dict(pages=4, kv_heads=2, head_dim=128), **kw})


def query(**kw):
    return lce.KV8QueryDesc(**{**dict(tokens=3, q_heads=8, seqs=2, table_width=5, type=2, causal=1,
                                      window=0, max_q=0, max_len=0, scale=0.1, softcap=0.0,
                                      q_token_stride=1024, q_head_stride=128), **kw})


def size(c):
    n = ctypes.c_int64()
    st = lce.lib().lce_kv8_cache_size(ctypes.byref(c), ctypes.byref(n))
    return st, n.value


def test_desc_layouts_match_header():
    assert ctypes.sizeof(lce.KV8CacheDesc) == 12
    assert ctypes.sizeof(lce.KV8QueryDesc) == 9 * 4 + 8 + 4 + 16      # the int64s are aligned
    assert ctypes.sizeof(lce.RotaryDesc) == 28
    assert ctypes.sizeof(lce.RotaryRows) == 4 + 4 + 16 + 32


def test_cache_size():
    for dim in (64, 128, 256):
        assert size(cache(head_dim=dim)) == (lce.LCE_OK, 4 * 2 * (128 * dim + 128))
    assert size(cache(pages=2 ** 31 - 1, kv_heads=8))[1] == (2 ** 31 - 1) * 8 * 129 * 128
    assert lce.lib().lce_kv8_cache_size(ctypes.byref(cache()), None) == lce.LCE_EINVAL
    assert lce.lib().lce_kv8_cache_size(None, ctypes.byref(ctypes.c_int64())) == lce.LCE_EINVAL


def call_append(c=None, data=P, type=2, k=P, ks=(256, 128), v=P, vs=(256, 128), n=3, seqs=2,
                width=5, table=P, start=P, lengths=P):
    return lce.lib().lce_kv8_append(ctypes.byref(c or cache()), data, type, k, *ks, v, *vs, n, seqs,
                                    width, table, start, lengths, None)


def call_read(c=None, data=P, slots=P, n=3, type=2, k=P, v=P):
    return lce.lib().lce_kv8_read(ctypes.byref(c or cache()), data, slots, n, type, k, v, None)


def call_attention(c=None, q=None, data=P, qp=P, table=P, start=P, lengths=P, slopes=None,
                   prefix=None, out=P, lse=None, ws=P, n=BIG):
    return lce.lib().lce_kv8_attention(ctypes.byref(c or cache()), data,
                                       ctypes.byref(q or query()), qp, table, start, lengths, slopes,
                                       prefix, out, lse, ws, n, None)


@pytest.mark.parametrize("field,value,status", [
    ("pages", 0, "LCE_EINVAL"), ("kv_heads", 0, "LCE_EINVAL"), ("kv_heads", -1, "LCE_EINVAL"),
    ("head_dim", 96, "LCE_EUNSUPPORTED"), ("head_dim", 0, "LCE_EUNSUPPORTED"),
    ("kv_heads", 65536, "LCE_EUNSUPPORTED")])
def test_cache_desc_refusals(field, value, status):
    c = cache(**{field: value})
    assert size(c)[0] == getattr(lce, status)
    assert lce.last_error()
    for call in (call_append, call_read, call_attention):
        assert call(c) == getattr(lce, status)


def test_append_refusals():
    assert call_append(n=0, data=None, k=None, v=None, table=None) == lce.LCE_OK
    for kw, status in ((dict(n=-1), lce.LCE_EINVAL), (dict(type=3), lce.LCE_EINVAL),
                       (dict(seqs=0), lce.LCE_EINVAL), (dict(width=0), lce.LCE_EINVAL),
                       (dict(width=2 ** 24 + 1), lce.LCE_EUNSUPPORTED),
                       (dict(c=cache(kv_heads=65535), n=2 ** 31 - 1), lce.LCE_EUNSUPPORTED),
                       (dict(seqs=2 ** 31 - 1), lce.LCE_EUNSUPPORTED),
                       (dict(ks=(257, 128)), lce.LCE_EALIGN), (dict(vs=(256, 132)), lce.LCE_EALIGN),
                       (dict(type=0, ks=(258, 128)), lce.LCE_EALIGN)):
        assert call_append(**kw) == status, kw
        assert lce.last_error()
    for name in ("data", "k", "v", "table", "start", "lengths"):
        assert call_append(**{name: None}) == lce.LCE_EINVAL
        assert call_append(**{name: P + 2}) == lce.LCE_EALIGN


def test_read_refusals():
    assert call_read(n=0, data=None, k=None, v=None, slots=None) == lce.LCE_OK
    assert call_read(n=-1) == lce.LCE_EINVAL
    assert call_read(n=2 ** 31) == lce.LCE_EINVAL
    assert call_read(c=cache(kv_heads=65535), n=2 ** 31 - 1) == lce.LCE_EUNSUPPORTED
    assert call_read(type=3) == lce.LCE_EINVAL
    for name in ("data", "k", "v", "slots"):
        assert call_read(**{name: None}) == lce.LCE_EINVAL
        assert call_read(**{name: P + 4}) == lce.LCE_EALIGN


def test_attention_refusals():
    for field, value, status in (
            ("tokens", -1, lce.LCE_EINVAL), ("seqs", 0, lce.LCE_EINVAL),
            ("table_width", 0, lce.LCE_EINVAL), ("q_heads", 0, lce.LCE_EINVAL),
            ("q_heads", 7, lce.LCE_EINVAL), ("type", 0, lce.LCE_EUNSUPPORTED),
            ("type", 9, lce.LCE_EINVAL), ("causal", 2, lce.LCE_EINVAL),
            ("window", -1, lce.LCE_EINVAL), ("max_q", -1, lce.LCE_EINVAL),
            ("max_len", -1, lce.LCE_EINVAL), ("scale", 0.0, lce.LCE_EINVAL),
            ("scale", float("nan"), lce.LCE_EINVAL), ("scale", 3e38, lce.LCE_EINVAL),
            ("softcap", -1.0, lce.LCE_EINVAL), ("softcap", float("nan"), lce.LCE_EINVAL),
            ("softcap", float("inf"), lce.LCE_EINVAL), ("softcap", 1e-31, lce.LCE_EINVAL),
            ("table_width", 2 ** 26, lce.LCE_EUNSUPPORTED),
            ("tokens", 2 ** 28, lce.LCE_EUNSUPPORTED), ("seqs", 2 ** 28, lce.LCE_EUNSUPPORTED),
            ("q_token_stride", 1025, lce.LCE_EALIGN), ("q_head_stride", 4, lce.LCE_EALIGN)):
        assert call_attention(q=query(**{field: value})) == status, (field, value)
        assert lce.last_error()
    assert call_attention(q=query(tokens=0), data=None, qp=None, out=None, ws=None) == lce.LCE_OK
    for name in ("data", "qp", "out", "ws"):
        assert call_attention(**{name: None}) == lce.LCE_EINVAL
        assert call_attention(**{name: P + 8}) == lce.LCE_EALIGN
    for name in ("table", "start", "lengths"):
        assert call_attention(**{name: None}) == lce.LCE_EINVAL
    for name in ("table", "start", "lengths", "slopes", "prefix", "lse"):
        assert call_attention(**{name: P + 2}) == lce.LCE_EALIGN
    assert call_attention(n=100) == lce.LCE_EINVAL
    assert "workspace" in lce.last_error()


def test_workspace_serves_fewer_tokens_and_any_options():
    def need(c=None, **kw):
        n = ctypes.c_int64()
        assert lce.lib().lce_kv8_workspace_size(ctypes.byref(c or cache()), ctypes.byref(query(**kw)),
                                                ctypes.byref(n)) == lce.LCE_OK
        return n.value
    assert need() > lce.KV8_WORKSPACE_ZERO
    assert need(max_q=7, max_len=9, window=3, causal=0, softcap=2.0) == need()
    for width in (1, 5, 4096):
        sizes = [need(tokens=t, table_width=width) for t in (0, 1, 2, 7, 100, 5000, 10 ** 6)]
        assert sizes == sorted(sizes)
    for dim, most in ((64, 18), (128, 36), (256, 69)):
        big = need(cache(head_dim=dim), tokens=10 ** 6, table_width=4096)
        assert big - lce.KV8_WORKSPACE_ZERO <= most * 10 ** 6
    n = ctypes.c_int64()
    assert lce.lib().lce_kv8_workspace_size(ctypes.byref(cache()), None, ctypes.byref(n)) == \
        lce.LCE_EINVAL
    assert lce.lib().lce_kv8_workspace_size(ctypes.byref(cache()), ctypes.byref(query()), None) == \
        lce.LCE_EINVAL


def test_binding_refuses_before_it_calls():
    for call in (lambda: lce.kv8_append(None, None, None, None, None, None),
                 lambda: lce.kv8_read(None, None), lambda: lce.kv8_attention(None, None, None, None, None),
                 lambda: lce.kv8_workspace(None, None, None), lambda: lce.rotary(None, None, None)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        lce.KV8Cache(2, 64)
    with pytest.raises(ValueError):
        lce.KV8Cache(2, 64, pages=3, device="cpu")
    with pytest.raises(ValueError):
        lce.KV8Cache(2, 64, data=torch.zeros(3, 2, 129 * 64, dtype=torch.uint8))  # not on a device
    for kw in (dict(head_dim=1), dict(head_dim=8, rot_dim=3), dict(head_dim=8, rot_dim=10),
               dict(head_dim=8, scaling="other"), dict(head_dim=8, freqs=[1.0]),
               dict(head_dim=4, freqs=[1.0, 2.0], scaling="linear"), dict(head_dim=8, device="cpu"),
               dict(head_dim=1 << 40)):
        with pytest.raises(ValueError):
            lce.Rotary(**kw)
    for kw in (dict(base=1.0), dict(base=float("inf")), dict(scaling="linear", factor=0.5),
               dict(scaling="ntk", factor=float("nan")), dict(scaling="yarn", factor=2.0, original=0),
               dict(freqs=[1.0, float("inf"), 0.0, 0.0])):
        with pytest.raises(lce.LceError):
            lce.Rotary(8, **kw)


# ---- rotary positions

def frequencies(rot, base=10000.0, scaling=0, factor=1.0, original=4096.0):
    out, scale = (ctypes.c_double * (rot // 2))(), ctypes.c_float()
    assert lce.lib().lce_rotary_frequencies(rot, base, scaling, factor, original, out,
                                            ctypes.byref(scale)) == lce.LCE_OK
    return np.array(out[:]), scale.value


def test_frequencies():
    plain, scale = frequencies(64)
    assert np.allclose(plain, 10000.0 ** (-np.arange(32) / 32), rtol=1e-14, atol=0) and scale == 1
    assert np.allclose(frequencies(64, scaling=1, factor=8.0)[0], plain / 8, rtol=1e-14, atol=0)
    # ntk: the slowest pair becomes factor times as slow, the fastest stays
    ntk = frequencies(64, scaling=2, factor=8.0)[0]
    assert ntk[0] == 1 and math.isclose(ntk[-1], plain[-1] / 8, rel_tol=1e-12)
    # yarn: fast pairs stay, slow ones become factor times as slow, one way between
    yarn, scale = frequencies(128, scaling=3, factor=4.0)
    turns = 4096 * frequencies(128)[0] / (2 * math.pi)
    ratio = frequencies(128)[0] / yarn
    assert (ratio[turns > 34] == 1).all() and np.allclose(ratio[turns < 0.8], 4, rtol=1e-14)
    assert (np.diff(ratio) >= 0).all()
    assert math.isclose(scale, 0.1 * math.log(4) + 1, rel_tol=1e-6)
    assert frequencies(2, scaling=2, factor=3.0)[0].tolist() == [1.0]


def test_frequency_refusals():
    f, out, s = lce.lib().lce_rotary_frequencies, (ctypes.c_double * 8)(), ctypes.c_float()
    for args in ((0, 1e4, 0, 1, 1), (3, 1e4, 0, 1, 1), (65538, 1e4, 0, 1, 1), (4, 1.0, 0, 1, 1),
                 (4, float("nan"), 0, 1, 1), (4, 1e4, 4, 1, 1), (4, 1e4, -1, 1, 1),
                 (4, 1e4, 1, 0.9, 1), (4, 1e4, 3, 2, 0.5), (4, 1e300, 2, 1e20, 1)):
        assert f(*args, out, ctypes.byref(s)) == lce.LCE_EINVAL, args
    assert f(4, 1e4, 0, 1, 1, None, ctypes.byref(s)) == lce.LCE_EINVAL
    assert f(4, 1e4, 0, 1, 1, out, None) == lce.LCE_EINVAL


def test_turns_are_the_nearest_64_bit_fractions():
    values = [1.0, 0.5, 1e-4, 1e-30, 0.0, -1.0, 7.0, 2 * math.pi, -1e-30, 12345.678]
    a, out = (ctypes.c_double * len(values))(*values), (ctypes.c_uint64 * len(values))()
    assert lce.lib().lce_rotary_turns(a, len(values), out) == lce.LCE_OK
    for x, got in zip(values, out):
        want = Fraction(x) / (2 * ref.PI) * 2 ** 64
        # the quotient in 64 bits, and its rounding: two of the last places that whole turns leave
        off = (got - want) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= 1 + 2 * abs(x), x
    assert lce.lib().lce_rotary_turns(a, 0, out) == lce.LCE_EINVAL
    assert lce.lib().lce_rotary_turns(None, 1, out) == lce.LCE_EINVAL


def rows(**kw):
    return lce.RotaryRows(**{**dict(heads=4, x=P, y=P, x_token_stride=256, x_head_stride=64,
                                    y_token_stride=256, y_head_stride=64), **kw})


def call_rotary(q=None, k=None, turns=P, positions=P, **kw):
    d = lce.RotaryDesc(**{**dict(tokens=3, head_dim=64, rot_dim=64, type=2, interleaved=0, backward=0,
                                 scale=1.0), **kw})
    return lce.lib().lce_rotary(ctypes.byref(d), turns, positions,
                                ctypes.byref(q) if q is not None else None,
                                ctypes.byref(k) if k is not None else None, None)


def test_rotary_refusals():
    assert call_rotary(tokens=0, turns=None, positions=None) == lce.LCE_OK
    for kw in (dict(tokens=-1), dict(head_dim=1), dict(head_dim=65537), dict(rot_dim=0),
               dict(rot_dim=3), dict(rot_dim=66), dict(type=3), dict(interleaved=2),
               dict(backward=-1), dict(scale=float("inf")), dict(turns=None), dict(positions=None)):
        assert call_rotary(rows(), **kw) == lce.LCE_EINVAL, kw
        assert lce.last_error()
    assert call_rotary() == lce.LCE_EINVAL
    for bad in (rows(heads=0), rows(x=None), rows(y=None)):
        assert call_rotary(bad) == lce.LCE_EINVAL
        assert call_rotary(rows(), bad) == lce.LCE_EINVAL
    assert call_rotary(rows(x=P + 1)) == lce.LCE_EALIGN
    assert call_rotary(rows(), rows(y=P + 2), type=0) == lce.LCE_EALIGN
    assert call_rotary(rows(), turns=P + 4) == lce.LCE_EALIGN
    assert call_rotary(rows(), positions=P + 4) == lce.LCE_EALIGN
    assert call_rotary(rows(heads=1 << 21)) == lce.LCE_EUNSUPPORTED
    assert call_rotary(rows(heads=1 << 20), tokens=2 ** 31 - 1, head_dim=65536, rot_dim=65536) == \
        lce.LCE_EUNSUPPORTED
    assert lce.lib().lce_rotary(None, P, P, None, None, None) == lce.LCE_EINVAL


def test_rotary_refuses_rows_that_share_memory():
    for kw in (dict(y_head_stride=0), dict(y_head_stride=63), dict(y_token_stride=0),
               dict(y_token_stride=255), dict(y_token_stride=-255), dict(y_head_stride=-63),
               dict(y_head_stride=128, y_token_stride=64), dict(x_head_stride=128, x_token_stride=512),
               dict(y_head_stride=2 ** 63 - 1, y_token_stride=2 ** 63 - 1)):
        bad = rows(**kw)
        assert call_rotary(bad) == lce.LCE_EINVAL, kw
        assert call_rotary(rows(), bad) == lce.LCE_EINVAL, kw
    assert call_rotary(rows(heads=1, y=BIG, y_token_stride=63)) == lce.LCE_EINVAL


def test_yarn_needs_the_first_pairs_whole_turn():
    out, s = (ctypes.c_double * 8)(), ctypes.c_float()
    for original, want in ((6.0, lce.LCE_EINVAL), (7.0, lce.LCE_OK)):
        assert lce.lib().lce_rotary_frequencies(16, 1e4, 3, 4.0, original, out,
                                                ctypes.byref(s)) == want
    # every pair but the first, which turns 1.1 times, is slowed
    assert out[0] == 1 and np.allclose(out[1:], 1e4 ** (-np.arange(1, 8) / 8) / 4, rtol=1e-14)


@pytest.mark.parametrize("scale", [1e300, float("inf"), float("nan"), -1e39])
def test_rotary_scale_is_a_float32(scale):
    with pytest.raises(ValueError, match="scale"):
        lce.Rotary(8, scale=scale)


# ---- the oracle, pinned

def test_reference_codes_by_hand_worked_values():
    assert ref.E4M3[[0, 1, 7, 8, 0x38, 0x7E, 0x80]].tolist() == [0, 2 ** -9, 7 * 2 ** -9, 2 ** -6, 1,
                                                                448, 0]
    assert np.isnan(ref.E4M3[[0x7F, 0xFF]]).all()
    x = [17.0, 19.0, 18.0, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -10, 447.9, -0.0, 1.0625, 1.1875]
    assert ref.E4M3[ref.encode(x)].tolist() == [16, 20, 18, 0, 2 ** -8, 0, 448, 0, 1, 1.25]
    assert ref.encode([-0.0, -2.0 ** -10]).tolist() == [128, 128]
    for top, want in ((448, 0), (448.1, 1), (1.0, -8), (1.75, -8), (1.76, -7), (0, -126),
                      (3.4028234663852886e38, 120)):
        assert ref.scale_exponent(top) == want


def test_reference_appends_by_hand_worked_values():
    c = ref.Cache(1, 1, 64, 0)
    k = np.full((3, 1, 64), 448.0)
    k[1] = 1.0
    c.append([0], 3, k, k / 448)
    assert c.data[0, 0, 128 * 64] == 127 and c.data[0, 0, 128 * 64 + 4] == 127 - 8
    assert c.read(1)[0][0, 0] == 1.0
    # a fourth token 2^9 times as large: 1.0 becomes 1 / 512 of a scale of 512, a subnormal code
    c.append([0], 4, np.full((1, 1, 64), 448.0 * 512), np.zeros((1, 1, 64)))
    assert c.data[0, 0, 128 * 64] == 136 and c.read(1)[0][0, 0] == 1.0
    assert c.data[0, 0, 64] == 1
    # and another 2 times as large takes it to half of one, which rounds to even
    c.append([0], 5, np.full((1, 1, 64), 448.0 * 1024), np.zeros((1, 1, 64)))
    assert c.read(1)[0][0, 0] == 0.0 and c.read(0)[0][0, 0] == 448.0
