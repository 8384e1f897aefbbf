"""Integers past 32 bits given to the attention calls of the binding: they mean what they say, and are not cut to their low bits.  No GPU needed."""
import pytest
import torch

from paper_2202_01085_amd import f3m


def made(**more):
    how = dict(max_q=None, max_k=None, scale=0.5, causal=True, window=0, sinks=0)
    how.update(more)
    q = torch.zeros((6, 2, 32), dtype=torch.bfloat16)
    return f3m._attention_args(q, q.shape, f3m.Rows(), f3m.Rows(), f3m.Rows(), 2, 9, 9, None, None, **how)


@pytest.mark.parametrize("big", [2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1, 10 ** 30])
def test_large_numbers_are_as_good_as_none(big):
    a = made(window=big, sinks=big, max_q=big, max_k=big)
    assert a.window == a.sinks == 2 ** 31 - 1 and a.max_q == 6 and a.max_k == 9      # no sequence is longer than all rows


@pytest.mark.parametrize("small", [-1, -2 ** 31, -2 ** 32, -2 ** 32 + 5])
def test_negative_numbers_stay_negative(small):
    a = made(window=small, sinks=small, max_q=small, max_k=small)
    assert a.window == a.sinks == a.max_q == a.max_k == -1


def test_others_are_taken_as_they_are():
    a = made(window=7, sinks=3, max_q=4, max_k=0)
    assert (a.window, a.sinks, a.max_q, a.max_k, a.total_q, a.total_k) == (7, 3, 4, 0, 6, 9)
    a = made()
    assert (a.max_q, a.max_k) == (6, 9)
