"""Host-side checks of the attention and cache calls: what is refused is refused before a device is touched.  No GPU needed."""
import ctypes
import os

import pytest
import torch

import attention_util as au
from paper_2202_01085_amd import build, f3m

INVALID, UNSUPPORTED = 1, 3
FAKE = 4096          # never dereferenced: every call below fails its checks, or has nothing to do


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(f3m.LIB_PATH):
        build.build_lib()
    return f3m.lib()


def args(**more):
    a = f3m.AttentionArgs(dtype=0, batch=1, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, max_q=10, max_k=10, total_q=10, total_k=10)
    a.q, a.k, a.v = f3m.Rows(FAKE, 256, 64), f3m.Rows(FAKE, 128, 64), f3m.Rows(FAKE, 128, 64)
    for n, x in more.items():
        setattr(a, n, x)
    return a


def cache(**more):
    c = f3m.CacheInfo(held=2, kv_heads=2, head_dim=64, page_size=16, pages=8, k=FAKE, v=FAKE, k_exp=FAKE, v_exp=FAKE)
    for n, x in more.items():
        setattr(c, n, x)
    return c


OUT, KV = f3m.Rows(FAKE, 256, 64), f3m.Rows(FAKE, 128, 64)

BAD = [(dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(heads=0), INVALID), (dict(heads=3), INVALID), (dict(kv_heads=0), INVALID),
       (dict(head_dim=0), INVALID), (dict(head_dim=60), INVALID), (dict(head_dim=136), UNSUPPORTED), (dict(batch=-1), INVALID),
       (dict(max_q=-1), INVALID), (dict(max_k=-1), INVALID), (dict(total_q=-1), INVALID), (dict(total_k=-1), INVALID),
       (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(window=4, causal=0), INVALID), (dict(sinks=4), INVALID),
       (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=-1.0), INVALID),
       (dict(batch=2), INVALID), (dict(q_offsets=FAKE), INVALID), (dict(total_q=2 ** 31), UNSUPPORTED), (dict(total_k=2 ** 31 - 1), UNSUPPORTED),
       (dict(max_q=2 ** 30), UNSUPPORTED), (dict(batch=2 ** 23, q_offsets=FAKE, k_offsets=FAKE), UNSUPPORTED)]


@pytest.mark.parametrize("more,status", BAD)
def test_arguments_that_are_refused(lib, more, status):
    a = args(**more)
    if "max_q" in more and status == UNSUPPORTED:
        a.max_q = 2 ** 31 - 1
    ref = ctypes.byref(a)
    assert lib.f3m_attention(ref, ctypes.byref(OUT), FAKE, FAKE, 1 << 40, None) == status
    assert lib.f3m_last_error() != b""
    r = [ctypes.byref(x) for x in (OUT, OUT, OUT, KV, KV)]
    assert lib.f3m_attention_grad(ref, r[0], r[1], FAKE, r[2], r[3], r[4], FAKE, 1 << 40, None) == status
    assert lib.f3m_attention_grad_workspace(ref) == -status
    if more != dict(q_offsets=FAKE):     # all that a call over a cache needs
        assert lib.f3m_attention_workspace(ref) == -status


def test_tensors_that_are_refused(lib):
    out, big = ctypes.byref(OUT), 1 << 40
    ok = ctypes.byref(args())
    assert lib.f3m_attention(None, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_attention(ok, None, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_attention(ok, out, None, FAKE, big, None) == INVALID
    for name in ("q", "k", "v"):
        for rows in (f3m.Rows(None, 256, 64), f3m.Rows(FAKE + 2, 256, 64), f3m.Rows(FAKE, 252, 64), f3m.Rows(FAKE, 256, 60), f3m.Rows(FAKE, -256, 64)):
            assert lib.f3m_attention(ctypes.byref(args(**{name: rows})), out, FAKE, FAKE, big, None) == INVALID
    for rows in (f3m.Rows(FAKE, 0, 64), f3m.Rows(FAKE, 256, 0), f3m.Rows(FAKE, 128, 64), f3m.Rows(FAKE, 64, 512), f3m.Rows(FAKE, 56, 2560)):
        assert lib.f3m_attention(ok, ctypes.byref(rows), FAKE, FAKE, big, None) == INVALID        # written rows overlap
    # many keys, one row: the call works in parts and needs its workspace
    a = args(max_q=1, total_q=1, max_k=100000, total_k=100000)
    need = lib.f3m_attention_workspace(ctypes.byref(a))
    assert need > 0 and need % 4 == 0
    assert lib.f3m_attention(ctypes.byref(a), out, FAKE, FAKE, need - 1, None) == INVALID
    assert lib.f3m_attention(ctypes.byref(a), out, FAKE, None, need, None) == INVALID
    assert lib.f3m_attention(ctypes.byref(a), out, FAKE, FAKE + 4, need, None) == INVALID
    r = [ctypes.byref(x) for x in (OUT, OUT, OUT, KV, KV)]
    need = lib.f3m_attention_grad_workspace(ok)
    assert need == 4 * 128
    assert lib.f3m_attention_grad(ok, r[0], r[1], FAKE, r[2], r[3], r[4], FAKE, need - 1, None) == INVALID
    assert lib.f3m_attention_grad(ok, r[0], r[1], None, r[2], r[3], r[4], FAKE, need, None) == INVALID
    assert lib.f3m_attention_grad(ok, None, r[1], FAKE, r[2], r[3], r[4], FAKE, need, None) == INVALID
    assert lib.f3m_attention_grad(ok, r[0], r[1], FAKE, r[2], None, r[4], FAKE, need, None) == INVALID
    assert lib.f3m_attention_grad(ok, r[0], r[1], FAKE, r[2], ctypes.byref(f3m.Rows(FAKE, 128, 0)), r[4], FAKE, need, None) == INVALID
    # nothing to do: no device is needed
    assert lib.f3m_attention(ctypes.byref(args(total_q=0, max_q=0)), None, None, None, 0, None) == 0
    assert lib.f3m_attention(ctypes.byref(args(batch=0, q_offsets=FAKE, k_offsets=FAKE)), out, FAKE, None, 0, None) == 0
    assert lib.f3m_attention_grad(ctypes.byref(args(batch=0, q_offsets=FAKE, k_offsets=FAKE)), *r[:2], FAKE, *r[2:], None, 0, None) == 0


@pytest.mark.parametrize("more,status", [(dict(held=3), INVALID), (dict(held=-1), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID),
                                         (dict(head_dim=72), UNSUPPORTED), (dict(head_dim=144), UNSUPPORTED), (dict(page_size=0), INVALID),
                                         (dict(page_size=4), INVALID), (dict(page_size=24), INVALID), (dict(page_size=2048), INVALID),
                                         (dict(pages=-1), INVALID), (dict(pages=2 ** 40), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
                                         (dict(k=FAKE + 8), INVALID), (dict(k_exp=None), INVALID), (dict(v_exp=None), INVALID)])
def test_caches_that_are_refused(lib, more, status):
    c = ctypes.byref(cache(**more))
    r = ctypes.byref(KV)
    assert lib.f3m_cache_write(c, 0, r, r, FAKE, 5, None) == status
    assert lib.f3m_cache_read(c, 0, r, r, FAKE, 5, None) == status
    assert lib.f3m_cache_attention(c, ctypes.byref(args()), FAKE, 4, 4, FAKE, ctypes.byref(OUT), FAKE, FAKE, 1 << 40, None) == status


@pytest.mark.parametrize("more", [dict(k_exp=FAKE + 2), dict(v_exp=FAKE + 1)])
def test_exponents_are_read_in_words(lib, more):
    c, r = ctypes.byref(cache(**more)), ctypes.byref(KV)
    assert lib.f3m_cache_write(c, 0, r, r, FAKE, 5, None) == INVALID
    assert lib.f3m_cache_attention(c, ctypes.byref(args()), FAKE, 4, 4, FAKE, ctypes.byref(OUT), FAKE, FAKE, 1 << 40, None) == INVALID


def test_cache_calls_that_are_refused(lib):
    c, r, ok, out = ctypes.byref(cache()), ctypes.byref(KV), ctypes.byref(args()), ctypes.byref(OUT)
    for call in (lib.f3m_cache_write, lib.f3m_cache_read):
        assert call(None, 0, r, r, FAKE, 5, None) == INVALID
        assert call(c, 2, r, r, FAKE, 5, None) == INVALID
        assert call(c, 0, None, r, FAKE, 5, None) == INVALID
        assert call(c, 0, r, r, None, 5, None) == INVALID
        assert call(c, 0, r, r, FAKE, -1, None) == INVALID
        assert call(c, 0, r, ctypes.byref(f3m.Rows(FAKE + 8, 128, 64)), FAKE, 5, None) == INVALID
        assert call(ctypes.byref(cache(held=1)), 0, r, r, FAKE, 5, None) == INVALID
        assert call(c, 0, None, None, None, 0, None) == 0
    assert lib.f3m_cache_read(c, 0, ctypes.byref(f3m.Rows(FAKE, 128, 0)), r, FAKE, 5, None) == INVALID
    big = 1 << 40
    assert lib.f3m_cache_attention(None, ok, FAKE, 4, 4, FAKE, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(c, None, FAKE, 4, 4, FAKE, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(c, ok, None, 4, 4, FAKE, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(c, ok, FAKE, 3, 4, FAKE, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(c, ok, FAKE, 4, -1, FAKE, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(c, ok, FAKE, 4, 4, None, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(c, ok, FAKE, 2 ** 30, 2 ** 30, FAKE, out, FAKE, FAKE, big, None) == UNSUPPORTED
    assert lib.f3m_cache_attention(ctypes.byref(cache(held=1)), ok, FAKE, 4, 4, FAKE, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(ctypes.byref(cache(kv_heads=4)), ok, FAKE, 4, 4, FAKE, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(ctypes.byref(cache(head_dim=32)), ok, FAKE, 4, 4, FAKE, out, FAKE, FAKE, big, None) == INVALID
    assert lib.f3m_cache_attention(c, ctypes.byref(args(total_q=0)), FAKE, 4, 4, FAKE, None, None, None, 0, None) == 0


def test_rows_read_from_a_cache_do_not_overlap(lib):
    c, ok = ctypes.byref(cache()), ctypes.byref(KV)
    for rows in (f3m.Rows(FAKE, 64, 64), f3m.Rows(FAKE, 64, 128), f3m.Rows(FAKE, 128, 120)):      # 5 rows of 2 heads of 64
        assert lib.f3m_cache_read(c, 0, ctypes.byref(rows), ok, FAKE, 5, None) == INVALID
        assert lib.f3m_cache_read(c, 0, ok, ctypes.byref(rows), FAKE, 5, None) == INVALID


def test_pages_past_32_bits_are_refused(lib):
    c, r = ctypes.byref(cache(kv_heads=2 ** 21, page_size=1024)), ctypes.byref(KV)
    assert lib.f3m_cache_write(c, 0, r, r, FAKE, 5, None) == UNSUPPORTED


def test_joins_of_more_blocks_than_a_grid_has_are_refused(lib):
    one = dict(heads=1, kv_heads=1)
    a = ctypes.byref(args(max_q=1, max_k=100000, total_q=2 ** 27, total_k=100000, **one))
    assert lib.f3m_attention(a, ctypes.byref(OUT), FAKE, FAKE, 1 << 60, None) == UNSUPPORTED
    a = ctypes.byref(args(batch=2 ** 20, q_offsets=FAKE, k_offsets=FAKE, window=1, sinks=1, max_q=512, max_k=128, total_q=2 ** 20, total_k=2 ** 20, **one))
    r = [ctypes.byref(x) for x in (OUT, OUT, OUT, KV, KV)]
    assert lib.f3m_attention_grad(a, r[0], r[1], FAKE, r[2], r[3], r[4], FAKE, 1 << 60, None) == UNSUPPORTED


def test_host_tensors_are_refused():
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        f3m.attention(x, x, x)
    with pytest.raises(TypeError):
        f3m.attention_grad(x, x, x, x, x, None)
    with pytest.raises(TypeError):
        f3m.KVCache(torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16))


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(f3m.Rows) == 24
    assert ctypes.sizeof(f3m.AttentionArgs) == 8 * 4 + 4 + 2 * 4 + 4 + 2 * 8 + 2 * 8 + 3 * 24
    assert ctypes.sizeof(f3m.CacheInfo) == 4 * 4 + 8 + 4 * 8


def test_the_reference_agrees_with_a_hand_computed_row():
    """two keys, scores 0 and log 3: weights 1/4 and 3/4"""
    q, k, v = (torch.tensor(x, dtype=torch.float64) for x in ([[1.0]], [[0.0], [1.0986122886681098]], [[4.0], [8.0]]))
    r = au.sequence(q, k, v, au.visible(1, 2, True, 0, 0), 1.0, 2.0 ** -8, False, dout=torch.ones((1, 1)).double())
    assert abs(r["out"].item() - 7.0) < 1e-12 and abs(r["lse"].item() - 1.3862943611198906) < 1e-12
    assert torch.allclose(r["dv"], torch.tensor([[0.25], [0.75]]).double()) and torch.allclose(r["dk"], torch.tensor([[-0.75], [0.75]]).double())
    assert au.visible(3, 5, True, 2, 1).int().tolist() == [[1, 1, 1, 0, 0], [1, 0, 1, 1, 0], [1, 0, 0, 1, 1]]
