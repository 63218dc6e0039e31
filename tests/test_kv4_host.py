"""Host side of the 4-bit cache's entry points, on the CPU: sizes and refusals.  Nothing is
ever launched; fake non-null pointers are plain integers."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from paper_2011_09398_amd import build as lce_build
from tests import kv4_util as ref

P = 0x10000
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def built():
    if lce_build.is_stale():
        lce_build.build()


def cache(**kw):
    return lce.KV4CacheDesc(**{**dict(pages=4, kv_heads=2, head_dim=128), **kw})


def query(**kw):
    return lce.KV4QueryDesc(**{**dict(tokens=3, q_heads=8, seqs=2, table_width=5, type=2, causal=1,
                                      window=0, list=0, max_q=0, max_len=0, scale=0.1,
                                      q_token_stride=1024, q_head_stride=128), **kw})


def size(c):
    n = ctypes.c_int64()
    st = lce.lib().lce_kv4_cache_size(ctypes.byref(c), ctypes.byref(n))
    return st, n.value


def test_desc_layouts_match_header():
    assert ctypes.sizeof(lce.KV4CacheDesc) == 12
    assert ctypes.sizeof(lce.KV4QueryDesc) == 10 * 4 + 4 + 4 + 16     # the int64s are aligned


def test_cache_size():
    for dim in (64, 128, 256):
        assert size(cache(head_dim=dim)) == (lce.LCE_OK, 4 * 2 * 76 * dim)
    assert size(cache(pages=2 ** 31 - 1, kv_heads=8))[1] == (2 ** 31 - 1) * 8 * 76 * 128
    assert lce.lib().lce_kv4_cache_size(ctypes.byref(cache()), None) == lce.LCE_EINVAL
    assert lce.lib().lce_kv4_cache_size(None, ctypes.byref(ctypes.c_int64())) == lce.LCE_EINVAL


@pytest.mark.parametrize("field,value,status", [
    ("pages", 0, "LCE_EINVAL"), ("kv_heads", 0, "LCE_EINVAL"), ("kv_heads", -1, "LCE_EINVAL"),
    ("head_dim", 96, "LCE_EUNSUPPORTED"), ("head_dim", 0, "LCE_EUNSUPPORTED"),
    ("kv_heads", 65536, "LCE_EUNSUPPORTED")])
def test_cache_desc_refusals(field, value, status):
    c = cache(**{field: value})
    assert size(c)[0] == getattr(lce, status)
    assert lce.last_error()
    assert call_append(c) == getattr(lce, status)
    assert call_attention(c) == getattr(lce, status)


def call_append(c=None, data=P, type=2, k=P, ks=(256, 128), v=P, vs=(256, 128), slots=P, n=3):
    return lce.lib().lce_kv4_append(ctypes.byref(c or cache()), data, type, k, *ks, v, *vs, slots,
                                    n, None)


def call_read(c=None, data=P, slots=P, n=3, type=2, k=P, v=P):
    return lce.lib().lce_kv4_read(ctypes.byref(c or cache()), data, slots, n, type, k, v, None)


def test_append_and_read_refusals():
    for call in (call_append, call_read):
        assert call(n=0, data=None, k=None, v=None, slots=None) == lce.LCE_OK
        assert call(n=-1) == lce.LCE_EINVAL
        assert call(n=2 ** 31) == lce.LCE_EINVAL
        assert call(c=cache(kv_heads=65535), n=2 ** 31 - 1) == lce.LCE_EUNSUPPORTED
        assert call(type=3) == lce.LCE_EINVAL
        for name in ("data", "k", "v", "slots"):
            assert call(**{name: None}) == lce.LCE_EINVAL
            assert call(**{name: P + 4}) == lce.LCE_EALIGN
    assert call_append(ks=(257, 128)) == lce.LCE_EALIGN
    assert call_append(vs=(256, 132)) == lce.LCE_EALIGN
    assert call_append(type=0, ks=(258, 128)) == lce.LCE_EALIGN
    assert "16 bytes" in lce.last_error()


def call_attention(c=None, q=None, data=P, qp=P, table=P, start=P, lengths=P, pages=None, out=P,
                   lse=None, ws=P, n=BIG):
    return lce.lib().lce_kv4_attention(ctypes.byref(c or cache()), data,
                                       ctypes.byref(q or query()), qp, table, start, lengths, pages,
                                       out, lse, ws, n, None)


def call_select(c=None, q=None, data=P, qp=P, table=P, start=P, lengths=P, first=1, last=1, out=P,
                ws=P, n=BIG):
    return lce.lib().lce_kv4_select(ctypes.byref(c or cache()), data,
                                    ctypes.byref(q or query(list=3)), qp, table, start, lengths,
                                    first, last, out, ws, n, None)


@pytest.mark.parametrize("call,base", [(call_attention, {}), (call_select, {"list": 3})])
def test_query_refusals(call, base):
    for field, value, status in (
            ("tokens", -1, lce.LCE_EINVAL), ("seqs", 0, lce.LCE_EINVAL),
            ("table_width", 0, lce.LCE_EINVAL), ("q_heads", 0, lce.LCE_EINVAL),
            ("q_heads", 7, lce.LCE_EINVAL), ("type", 0, lce.LCE_EUNSUPPORTED),
            ("type", 9, lce.LCE_EINVAL), ("causal", 2, lce.LCE_EINVAL),
            ("window", -1, lce.LCE_EINVAL), ("list", -1, lce.LCE_EINVAL),
            ("max_q", -1, lce.LCE_EINVAL), ("max_len", -1, lce.LCE_EINVAL),
            ("table_width", 2 ** 26, lce.LCE_EUNSUPPORTED),
            ("tokens", 2 ** 28, lce.LCE_EUNSUPPORTED), ("seqs", 2 ** 28, lce.LCE_EUNSUPPORTED),
            ("q_token_stride", 1025, lce.LCE_EALIGN), ("q_head_stride", 4, lce.LCE_EALIGN)):
        assert call(q=query(**{**base, field: value})) == status, (field, value)
        assert lce.last_error()
    assert call(q=query(**base, tokens=0), data=None, qp=None, out=None, ws=None) == lce.LCE_OK
    for name in ("data", "qp", "out", "ws"):
        assert call(**{name: None}) == lce.LCE_EINVAL
    for name in ("data", "qp", "ws"):
        assert call(**{name: P + 8}) == lce.LCE_EALIGN
    for name in ("table", "start", "lengths"):
        assert call(**{name: None}) == lce.LCE_EINVAL
        assert call(**{name: P + 2}) == lce.LCE_EALIGN
    assert call(n=100) == lce.LCE_EINVAL
    assert "workspace" in lce.last_error()
    assert lce.lib().lce_kv4_workspace_size(ctypes.byref(cache()), None,
                                            ctypes.byref(ctypes.c_int64())) == lce.LCE_EINVAL


def test_attention_and_select_refusals():
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call_attention(q=query(scale=scale)) == lce.LCE_EINVAL
        assert "scale" in lce.last_error()
    assert call_attention(q=query(scale=3e38)) == lce.LCE_EINVAL       # times log2(e)
    one = dict(q_heads=1, q_token_stride=64, q_head_stride=64)
    wide = cache(kv_heads=1, head_dim=64)
    assert call_select(c=wide, q=query(list=1, tokens=2 ** 24, **one)) == lce.LCE_EUNSUPPORTED
    assert call_attention(c=wide, q=query(list=1, tokens=2 ** 24, **one), pages=P) == \
        lce.LCE_EUNSUPPORTED
    assert call_attention(q=query(list=2)) == lce.LCE_EINVAL
    assert call_attention(q=query(list=2), pages=P + 1) == lce.LCE_EALIGN
    assert call_attention(out=P + 8) == lce.LCE_EALIGN
    assert call_attention(lse=P + 2) == lce.LCE_EALIGN
    assert call_select(q=query(list=0)) == lce.LCE_EINVAL
    assert call_select(first=-1) == lce.LCE_EINVAL
    assert call_select(last=-1) == lce.LCE_EINVAL
    assert call_select(out=P + 2) == lce.LCE_EALIGN
    assert call_select(c=cache(kv_heads=1, head_dim=256), q=query(list=1, q_heads=256)) == \
        lce.LCE_EUNSUPPORTED


def test_workspace_covers_lists_and_ranks():
    def need(**kw):
        n = ctypes.c_int64()
        assert lce.lib().lce_kv4_workspace_size(ctypes.byref(cache()), ctypes.byref(query(**kw)),
                                                ctypes.byref(n)) == lce.LCE_OK
        return n.value
    assert need() > lce.KV4_WORKSPACE_ZERO
    assert need(list=1000, max_q=7, max_len=9, window=3, causal=0) == need()
    assert need(tokens=100000, table_width=4096) >= lce.KV4_WORKSPACE_ZERO + 100000 * 2 * 4096 * 2


def test_binding_refuses_before_it_calls():
    with pytest.raises(TypeError):
        lce.kv4_append(None, None, None, None)
    with pytest.raises(ValueError):
        lce.KV4Cache(2, 64)
    with pytest.raises(ValueError):
        lce.KV4Cache(2, 64, data=torch.zeros(3, 2, 76 * 64, dtype=torch.uint8))   # not on a device


def test_reference_quantises_by_hand_worked_values():
    """The oracle of the GPU tests, pinned: a group whose largest value is 7 has e = 0."""
    x = np.zeros(32)
    x[:12] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5.01, -0.2, 0.26, -0.0]
    codes, byte, fine = ref.quantise(x)
    assert byte.tolist() == [127] and fine.all()
    assert ref.values(codes, byte)[:12].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -6, 0, 0.5, 0]
    assert codes[9] == codes[11] == 8                                  # zeros keep their sign
    for top, want in ((1.0, 125), (0.999, 124), (8.0, 128), (2.0 ** -126, 0), (2.0 ** -140, 0),
                      (0.0, 0), (3e38, 252)):
        assert ref.quantise(np.full(32, top))[1][0] == want
    assert ref.quantise(np.full(32, np.inf))[1][0] == 255
