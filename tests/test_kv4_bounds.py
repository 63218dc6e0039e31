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
