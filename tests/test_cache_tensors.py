"""A KVCache keeps to the tensors it was made of: others in their place, or other memory under them, are refused."""
import pytest
import torch

from paper_2202_01085_amd import f3m

NAMES = ("k", "v", "k_exp", "v_exp")


def test_tensors_are_not_replaced():
    c = object.__new__(f3m.KVCache)           # no device here: the attributes alone
    c._tensors = tuple(torch.zeros(1) for _ in NAMES)
    for i, name in enumerate(NAMES):
        assert getattr(c, name) is c._tensors[i]
        with pytest.raises(AttributeError):
            setattr(c, name, torch.zeros(2))
        with pytest.raises(AttributeError):
            delattr(c, name)


def test_tensors_that_moved_are_refused():
    c = object.__new__(f3m.KVCache)
    c._tensors = torch.zeros(4), torch.zeros(4), None, None
    c._at, c._c = (c.k.data_ptr(), c.v.data_ptr(), None, None), f3m.CacheInfo()
    assert c._info() is c._c
    c.v.resize_(1 << 20)
    with pytest.raises(ValueError):
        c._info()
    c._tensors = torch.zeros(0), torch.zeros(0), None, None
    c._at = (c.k.data_ptr() or None, c.v.data_ptr() or None, None, None)
    assert c._info() is c._c


@pytest.mark.gpu
def test_a_cache_that_grows_is_a_new_one():
    dev = "cuda:0"
    c = f3m.KVCache.empty(2, 16, 1, 32, device=dev)
    x = torch.randn((40, 1, 32), device=dev).bfloat16()
    slots = torch.arange(40, device=dev)
    c.write(x, x, slots)
    with pytest.raises(AttributeError):
        c.k = torch.cat([c.k, c.k])
    k, v, ke, ve = (torch.cat([t.view(torch.uint8), t.view(torch.uint8)]) for t in (c.k, c.v, c.k_exp, c.v_exp))
    big = f3m.KVCache(k.view(c.k.dtype), v.view(c.k.dtype), ke, ve)
    assert torch.equal(big.read(slots[:32])[0], c.read(slots[:32])[0])
    big.write(x, x, slots)
    assert big.read(slots)[0][32:].any()
    c.k.resize_((8, 1, 16, 32))
    table, ln, q = torch.zeros((1, 1), dtype=torch.int32, device=dev), torch.ones(1, dtype=torch.int32, device=dev), x[:1]
    for call in (lambda: c.write(x, x, slots), lambda: c.read(slots), lambda: c.attention(q, table, ln)):
        with pytest.raises(ValueError):
            call()
