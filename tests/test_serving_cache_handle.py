"""KVCache: what can be changed of it, and that calls go by what it holds at the time (no GPU: data on the CPU, the descriptor is looked at)."""
import pytest
import torch

import paper_2503_01483_amd as kt


def _cache(**kw):
    return kt.KVCache(2, 64, 2, 64, kt.KT_KV_U8, device="cpu", **kw)


def test_other_data_in_its_place_is_what_a_call_gets():
    cache = _cache()
    other = torch.zeros_like(cache.data)
    cache.data = other
    assert cache.data is other
    cache._on(-1)                                   # (-1: where torch says that a tensor on the CPU is)
    assert cache.desc.data == other.data_ptr()
    for bad in (other[:-1], other.view(torch.int8), other.repeat(2)[::2]):
        with pytest.raises(ValueError):
            cache.data = bad
    assert cache.data is other


def test_data_that_has_moved_or_shrunk_since():
    cache = _cache()
    cache.data.set_(torch.zeros_like(cache.data))   # the same tensor, elsewhere
    cache._on(-1)
    assert cache.desc.data == cache.data.data_ptr()
    cache.data.resize_(16)
    with pytest.raises(ValueError):
        cache._on(-1)
    with pytest.raises(ValueError):
        _cache()._on(0)                             # on another device than the call


@pytest.mark.parametrize("name", ["n_pages", "page_size", "n_heads", "head_dim", "format"])
def test_its_shape_stays(name):
    """A call checks its operands against these; the kernels go by the descriptor."""
    cache = _cache()
    assert getattr(cache, name) == getattr(cache.desc, name)
    with pytest.raises(AttributeError):
        setattr(cache, name, 1)
