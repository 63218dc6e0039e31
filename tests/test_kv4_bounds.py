"""Bounds of the 4-bit cache's entry points, on the CPU: what a kernel could not count, or
would read as something else, is refused before anything is launched."""
import ctypes

import pytest

import paper_2011_09398_amd as lce
from tests.test_kv4_host import built, cache, call_attention, call_select, P, query  # noqa: F401


@pytest.mark.parametrize("count", [2 ** 24 + 1, 2 ** 31 - 1])
def test_lists_longer_than_a_table_can_be(count):
    """Kernels count a list's entries, some hundreds past its end, in 32 bits."""
    q = query(list=count)
    assert call_attention(q=q, pages=P) == lce.LCE_EUNSUPPORTED
    assert str(count) in lce.last_error()
    assert call_select(q=q) == lce.LCE_EUNSUPPORTED
    assert str(count) in lce.last_error()


def test_a_cache_is_on_a_device():
    """Its tensors' addresses go to kernels: a buffer on the host is refused, as data is."""
    for device in ("cpu", "meta"):
        with pytest.raises(ValueError, match="device"):
            lce.KV4Cache(2, 64, pages=1, device=device)


def sizes(c=None, **kw):
    """Bytes of workspace for attention, selection and both."""
    out = []
    for name in ("attention_workspace", "select_workspace", "workspace"):
        n = ctypes.c_int64()
        assert getattr(lce.lib(), f"lce_kv4_{name}_size")(
            ctypes.byref(c or cache()), ctypes.byref(query(**kw)), ctypes.byref(n)) == lce.LCE_OK
        out.append(n.value - lce.KV4_WORKSPACE_ZERO)
    return out


def test_attention_needs_no_room_for_ranks():
    """Its states are bounded, whatever the tokens and the table's width; a workspace for
    them is enough for it."""
    for dim in (64, 128, 256):
        for tokens, width in ((4096, 2048), (8192, 16384), (1, 20000), (100000, 4096)):
            c, kw = cache(kv_heads=8, head_dim=dim), dict(tokens=tokens, table_width=width)
            states, ranks, both = sizes(c, **kw)
            assert 0 < states <= 4096 * 16 * (dim + 4) * 4 and ranks == tokens * 8 * width * 2
            assert both == max(states, ranks)
            n = lce.KV4_WORKSPACE_ZERO + states
            # what is one byte short is refused before anything else could be
            assert call_attention(c, query(**kw), n=n - 1) == lce.LCE_EINVAL
            assert "workspace" in lce.last_error()
            n = lce.KV4_WORKSPACE_ZERO + ranks
            assert call_select(c, query(**kw, list=3), n=n - 1) == lce.LCE_EINVAL
            assert "workspace" in lce.last_error()


def test_a_workspace_is_as_small_as_the_call():
    assert sizes(tokens=1, table_width=1)[0] == 0           # nothing to join
    assert sizes(tokens=0)[0] == 0
    # 2 heads of 2 tiles, a state for each page
    assert sizes(tokens=1, seqs=1, table_width=5)[0] <= 2 * 2 * 5 * 128 * 132 * 4


def test_a_workspace_serves_fewer_tokens():
    for dim in (64, 128, 256):
        for width in (1, 2, 3, 100, 5000):
            last = (0, 0, 0)
            for tokens in (0, 1, 2, 7, 100, 500, 511, 513, 2000, 4096, 5000, 100000):
                now = sizes(cache(head_dim=dim), tokens=tokens, table_width=width)
                assert all(a >= b for a, b in zip(now, last))
                last = now
