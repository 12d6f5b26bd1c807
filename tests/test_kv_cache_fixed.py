"""A KVCache hands the library addresses that it took when it was made: its tensors
and sizes cannot be replaced or deleted under it (no GPU)."""
import copy

import pytest

torch = pytest.importorskip("torch")

import paper_2406_13868_amd as sdq  # noqa: E402
from paper_2406_13868_amd import _lib  # noqa: E402

PARTS = ("k", "v", "k_scale", "v_scale", "position", "weight")


class _OnGpu(torch.Tensor):
    """A CPU tensor that passes for a device tensor: a cache only takes addresses."""
    is_cuda = True

    def __deepcopy__(self, memo):
        return self.clone()


def _cache():
    new = lambda dt, *more: torch.zeros((4, 2, 8, *more), dtype=dt).as_subclass(_OnGpu)  # noqa: E731
    return sdq.KVCache(new(torch.float8_e4m3fn, 32), new(torch.float8_e4m3fn, 32), new(torch.float32), new(torch.float32), new(torch.int32),
                       new(torch.float32))


@pytest.mark.parametrize("name", PARTS)
def test_tensors_are_not_replaced_or_deleted(name):
    cache = _cache()
    before = getattr(cache, name)
    with pytest.raises(AttributeError, match="with_state"):
        setattr(cache, name, before.clone())
    with pytest.raises(AttributeError, match="with_state"):
        setattr(cache, name, None)
    with pytest.raises(AttributeError, match="with_state"):
        delattr(cache, name)
    assert getattr(cache, name) is before and getattr(cache._c, name) == before.data_ptr()


@pytest.mark.parametrize("name", ["pages", "heads", "page_size", "dim", "device"])
def test_sizes_are_not_replaced(name):
    cache = _cache()
    before = getattr(cache, name)
    with pytest.raises(AttributeError, match="fixed"):
        setattr(cache, name, before)
    with pytest.raises(AttributeError, match="fixed"):
        delattr(cache, name)
    assert getattr(cache, name) == before


def test_with_state_takes_the_new_addresses():
    cache = _cache()
    p, w = cache.position.clone(), cache.weight.clone()
    other = cache.with_state(p, w)
    assert other.position is p and other.weight is w and (other._c.position, other._c.weight) == (p.data_ptr(), w.data_ptr())
    assert other.k is cache.k and cache._c.weight == cache.weight.data_ptr()


def test_copies_have_addresses_of_their_own_tensors():
    cache = _cache()
    same, deep = copy.copy(cache), copy.deepcopy(cache)
    for c in (same, deep):
        assert isinstance(c, sdq.KVCache) and bytes(c._c)[48:] == bytes(cache._c)[48:]
        assert all(getattr(c._c, n) == getattr(c, n).data_ptr() for n in PARTS)
    assert all(getattr(same, n) is getattr(cache, n) for n in PARTS)
    assert all(getattr(deep, n) is not getattr(cache, n) for n in PARTS)
    assert _lib.sdq_kv_cache.pages.offset == 48


def test_a_subclass_keeps_attributes_of_its_own():
    class Named(sdq.KVCache):
        pass

    c = _cache()
    named = Named(c.k, c.v, c.k_scale, c.v_scale)
    named.name = "block 3"
    named.name = "block 4"
    assert named.name == "block 4"
