"""Arguments that require gradients: attention() warns that its results carry no graph, and computes what it computes without."""
import warnings

import pytest
import torch

from paper_2202_01085_amd import f3m


def test_the_warning():
    x, y = torch.zeros(2), torch.zeros(2, requires_grad=True)
    with pytest.warns(UserWarning, match="attention_grad"):
        f3m._no_graph("attention", x, y)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        f3m._no_graph("attention", x, x)
        with torch.no_grad():
            f3m._no_graph("attention", x, y)


@pytest.mark.gpu
def test_calls_that_warn():
    x = torch.randn((5, 2, 32), device="cuda:0").bfloat16()
    y = x.clone().requires_grad_()
    want = f3m.attention(x, x, x)
    for args in ((y, x, x), (x, y, x), (x, x, y)):
        with pytest.warns(UserWarning, match="no graph"):
            got = f3m.attention(*args)
        assert torch.equal(got[0], want[0]) and not got[0].requires_grad
    c = f3m.KVCache.empty(1, 16, 2, 32, device="cuda:0")
    table, ln = torch.zeros((1, 1), dtype=torch.int32, device="cuda:0"), torch.ones(1, dtype=torch.int32, device="cuda:0")
    with pytest.warns(UserWarning, match="no graph"):
        c.attention(y[:1], table, ln)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            f3m.attention(y, y, y)
            c.attention(y[:1], table, ln)
        f3m.attention_grad(x, y, y, y, *want)
