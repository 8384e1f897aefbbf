"""Bytes of workspace that the gradients ask for: in proportion to what is cut, whatever the batch, the window and the sinks.  No GPU needed."""
import ctypes
import os
import random

import pytest

from paper_2202_01085_amd import build, f3m

MB = 2 ** 20
FAKE = 4096          # offsets, never read on the host


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(f3m.LIB_PATH):
        build.build_lib()
    return f3m.lib()


def grad_bytes(lib, batch, heads, kv_heads, dim, max_q, max_k, total_q, total_k, causal=1, window=0, sinks=0):
    a = f3m.AttentionArgs(dtype=0, batch=batch, heads=heads, kv_heads=kv_heads, head_dim=dim, causal=causal, window=window, sinks=sinks, scale=0.1,
                          max_q=max_q, max_k=max_k, total_q=total_q, total_k=total_k, q_offsets=FAKE, k_offsets=FAKE)
    got = lib.f3m_attention_grad_workspace(ctypes.byref(a))
    assert got >= 0
    return got


@pytest.mark.parametrize("case,most", [
    # one long sequence with a window: no sinks, four, sixteen, thousands, more than there are keys
    ((1, 8, 1, 128, 49152, 49152, 49152, 49152, 1, 128, 0), 150), ((1, 16, 2, 64, 49152, 49152, 49152, 49152, 1, 64, 4), 200),
    ((1, 64, 8, 64, 8192, 8192, 8192, 8192, 1, 16, 16), 200), ((1, 16, 16, 128, 49152, 49152, 49152, 49152, 1, 128, 4096), 420),
    ((1, 16, 16, 128, 49152, 49152, 49152, 49152, 1, 128, 2 ** 31 - 1), 420),
    # one long sequence among short ones
    ((100, 1, 1, 128, 16384, 16384, 17968, 17968), 100), ((64, 1, 1, 128, 8192, 8192, 12224, 12224), 100), ((32, 4, 4, 128, 8192, 8192, 10176, 10176), 150),
    ((100, 1, 1, 128, 16384, 16384, 17968, 17968, 1, 128, 4), 150),
    # buffers with room for more rows than the sequences have
    ((1, 1, 1, 64, 6709, 6709, 2 ** 24, 2 ** 24), 200)])
def test_parts_take_no_more_than_they_need(lib, case, most):
    stats = 8 * case[6] * case[1]
    assert grad_bytes(lib, *case) - stats <= most * MB


def test_parts_of_any_shape_are_bounded(lib):
    """rows: at most 1023 parts of 128 rows; keys: of four rounds of blocks (256 places above a head size of 64, else 512), 128 keys of two
    gradients each, and of eight for those of the sinks; fp32"""
    rng = random.Random(5)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))   # noqa: E731
    for _ in range(20000):
        kv, group, dim, batch = log(1, 64), log(1, 32), 8 * rng.randint(1, 16), log(1, 3000)
        mq, mk = log(1, 200000), log(1, 200000)
        if kv * batch * mk // 128 * 2 > 2 ** 23 or kv * batch * mq * group // 128 > 2 ** 20:     # too many work items are refused
            continue
        tq, tk = (rng.randint(m, m * batch) for m in (mq, mk))
        causal = rng.random() < 0.8
        window = rng.choice([0, log(1, 100000)]) if causal else 0
        sinks = rng.choice([0, 1, 4, log(1, 10000), 2 ** 31 - 1]) if window else 0
        places, wide = (256 if dim > 64 else 512), 4 * dim
        most = 8 * tq * group * kv + 256 + max(1023 * 128 * wide, (4 + 8) * places * 256 * wide)
        case = (batch, group * kv, kv, dim, mq, mk, tq, tk, int(causal), window, sinks)
        assert grad_bytes(lib, *case) <= most, case


def test_no_sequences(lib):
    assert grad_bytes(lib, 0, 4, 2, 64, 10, 10, 10, 10) == 4 * 128
    assert grad_bytes(lib, 0, 4, 2, 64, 10, 10, 10, 10, 1, 3, 1) == 4 * 128
