"""f3m.attention and f3m.attention_grad against the definition in 64 bits (attention_util.py, with the tolerances): every combination of
type and head size, lengths about the sizes of tiles, masks that leave rows empty, strides, NaN in hidden places, graphs, streams."""
import numpy as np
import pytest
import torch

import attention_util as au
from paper_2202_01085_amd import f3m

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF = torch.bfloat16, torch.float16


def normal(shape, seed, type, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * size).to(type)


def dev_offsets(o):
    return torch.tensor(o, dtype=torch.int32, device=DEV)


def run(type, D, Hq, Hk, nq, nk=None, causal=True, window=0, sinks=0, grad=True, seed=1, size=1.0, gsize=1.0):
    nk = nq if nk is None else nk
    qo, ko = au.offsets(nq), au.offsets(nk)
    q, k, v = normal((qo[-1], Hq, D), seed, type, size), normal((ko[-1], Hk, D), seed + 1, type, size), normal((ko[-1], Hk, D), seed + 2, type)
    do = normal((qo[-1], Hq, D), seed + 3, type, gsize) if grad else None
    scale = 1.0 / D ** 0.5
    print("attention", type, D, Hq, Hk, nq, nk, causal, window, sinks, flush=True)
    want = au.batch(q, k, v, qo, ko, float(np.float32(scale)), causal, window, sinks, do)
    how = dict(q_offsets=dev_offsets(qo), k_offsets=dev_offsets(ko), max_q=max(nq), max_k=max(nk), scale=scale, causal=causal, window=window, sinks=sinks)
    qd, kd, vd = q.to(DEV), k.to(DEV), v.to(DEV)
    out, lse = f3m.attention(qd, kd, vd, **how)
    au.close(lse, want, "lse")
    au.close(out, want, "out")
    if grad:
        dq, dk, dv = f3m.attention_grad(do.to(DEV), qd, kd, vd, out, lse, **how)
        au.close(dv, want, "dv")
        au.close(dk, want, "dk")
        au.close(dq, want, "dq")


@pytest.mark.parametrize("type", [BF, HF])
@pytest.mark.parametrize("D", [8, 32, 40, 64, 80, 96, 128])
def test_head_sizes(type, D):
    run(type, D, 4, 2, [65, 1, 130], seed=D)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 513])
@pytest.mark.parametrize("group", [1, 3, 8])
def test_lengths(n, group):
    run(BF, 64, group, 1, [n], seed=n)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nq,nk", [([5, 70, 300], [300, 70, 5]), ([1, 0, 40], [900, 10, 0]), ([200], [201]), ([129, 64], [64, 1000])])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_that_differ(D, nq, nk, causal):
    """more queries than keys with causal order: the first rows see nothing"""
    run(HF if D == 64 else BF, D, 4, 2, nq, nk, causal=causal, seed=7)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (64, 4), (100, 64), (128, 70), (600, 2), (2 ** 31 - 1, 5)])
@pytest.mark.parametrize("D", [64, 128])
def test_window_and_sinks(window, sinks, D):
    run(BF, D, 4, 2, [400, 33], window=window, sinks=sinks, seed=window % 1000)
    run(HF, D, 3, 1, [150, 20], [500, 10], window=window, sinks=sinks, seed=window % 1000 + 5)


@pytest.mark.parametrize("nq,nk,group", [(1, 20000, 1), (1, 5000, 8), (3, 9001, 4), (70, 6000, 2), (300, 9000, 1)])
def test_long_keys_few_rows(nq, nk, group):
    """the key axis is cut into parts that are joined"""
    run(BF, 128, 2 * group, 2, [nq, 1], [nk, 77], seed=nq, grad=False)
    run(HF, 64, group, 1, [nq], [nk], window=3000, sinks=5, seed=nq + 3, grad=False)


@pytest.mark.parametrize("type", [BF, HF])
def test_large_scores_and_small_gradients(type):
    """scores of a hundred and more (weights of one key alone), and gradients of 1e-4, whose products leave fp16's range unscaled"""
    run(type, 64, 2, 2, [300], size=4.0, seed=11)
    run(type, 128, 2, 1, [1500], causal=False, gsize=1e-4, seed=12)
    run(type, 128, 2, 1, [300], gsize=200.0, seed=13)


def test_growing_scores():
    """scores that rise along the keys, so that the running maximum moves tile after tile"""
    n, D = 700, 64
    q = torch.ones((n, 1, D), dtype=BF)
    k = (torch.arange(n)[:, None, None] / 64.0 * torch.ones((1, 1, D))).to(BF)
    v = normal((n, 1, D), 3, BF)
    scale = 1.0 / 8
    want = au.batch(q, k, v, [0, n], [0, n], scale)
    out, lse = f3m.attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=scale)
    au.close(lse, want, "lse")
    au.close(out, want, "out")
    k = k.flip(0).contiguous()
    want = au.batch(q, k, v, [0, n], [0, n], scale, causal=False)
    out, lse = f3m.attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=scale, causal=False)
    au.close(lse, want, "lse")
    au.close(out, want, "out")


def test_strides_and_rows_outside():
    """q, k, v as slices of one projection, results into slices; rows behind the last sequence and before the first stay as they are"""
    T, Hq, Hk, D = 210, 4, 2, 64
    x = normal((T, Hq + 2 * Hk, D + 8), 5, BF).to(DEV)
    q, k, v = x[:, :Hq, :D], x[:, Hq:Hq + Hk, :D], x[:, Hq + Hk:, :D]
    qo = [10, 100, 190]
    off = dev_offsets(qo)
    big = torch.full((Hq, T, 2 * D), 7.0, dtype=BF, device=DEV)
    out = big[:, :, D:].transpose(0, 1)
    lse = torch.full((T, Hq), 5.0, device=DEV)
    want = au.batch(q.cpu(), k.cpu(), v.cpu(), qo, qo, 0.125, window=50, sinks=2, dout=q.cpu())
    how = dict(q_offsets=off, k_offsets=off, max_q=90, max_k=90, scale=0.125, window=50, sinks=2)
    f3m.attention(q, k, v, out=out, lse=lse, **how)
    au.close(out, want, "out")
    au.close(lse, want, "lse")
    grads = [torch.full((T, h, D), 3.0, dtype=BF, device=DEV) for h in (Hq, Hk, Hk)]
    f3m.attention_grad(q, q, k, v, out, lse, dq=grads[0], dk=grads[1], dv=grads[2], **how)
    for y, name in zip(grads, ("dq", "dk", "dv")):
        au.close(y, want, name)
    torch.cuda.synchronize()
    assert (big[:, :, :D] == 7).all() and (lse[:10] == 5).all() and (lse[190:] == 5).all()
    assert (out[:10] == 7).all() and (out[190:] == 7).all()
    for y in grads:
        assert (y[:10] == 3).all() and (y[190:] == 3).all()


def test_broadcast_inputs():
    """one key head for all sequences' rows as stride 0 along the heads; its gradients come per head"""
    n, D = 90, 64
    q, k = normal((n, 2, D), 1, BF), normal((n, 1, D), 2, BF)
    wide = k.to(DEV).expand(n, 2, D)
    want = au.batch(q, k.expand(n, 2, D), k.expand(n, 2, D), [0, n], [0, n], 0.125, dout=q)
    out, lse = f3m.attention(q.to(DEV), wide, wide, scale=0.125)
    au.close(out, want, "out")
    dq, dk, dv = f3m.attention_grad(q.to(DEV), q.to(DEV), wide, wide, out, lse, scale=0.125)
    for y, name in zip((dq, dk, dv), ("dq", "dk", "dv")):
        au.close(y, want, name)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), "lowest"])
@pytest.mark.parametrize("type", [BF, HF])
def test_hidden_values_reach_nobody(bad, type):
    """the last 40 tokens hold NaN, infinities or the type's lowest value in k and v, as do q and dout there: tokens before them, and the
    gradients that come from those, are as if they were zeros"""
    n, cut, D = 333, 293, 64
    bad = torch.finfo(type).min if bad == "lowest" else bad
    q, k, v, do = (normal((n, h, D), i, type) for i, h in enumerate((4, 2, 2, 4)))
    do[cut:] = 0
    clean = au.batch(q[:cut], k[:cut], v[:cut], [0, cut], [0, cut], 0.125, window=100, sinks=2, dout=do[:cut])
    k[cut:, :, ::3] = bad
    v[cut:, :, 1::5] = bad
    for window, sinks, want in ((100, 2, clean), (0, 0, au.batch(q[:cut], k[:cut], v[:cut], [0, cut], [0, cut], 0.125))):
        out, lse = f3m.attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=0.125, window=window, sinks=sinks)
        au.close(out[:cut], want, "out")
        au.close(lse[:cut], want, "lse")
    out, lse = f3m.attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=0.125, window=100, sinks=2)
    dq, _, _ = f3m.attention_grad(do.to(DEV), q.to(DEV), k.to(DEV), v.to(DEV), out, lse, scale=0.125, window=100, sinks=2)
    au.close(dq[:cut], clean, "dq")


@pytest.mark.parametrize("type", [BF, HF])
def test_hidden_queries_reach_no_key(type):
    """tokens 0 .. 39 hold NaN in q and dout: with causal order and a window of 50, keys from 40 on do not depend on them; and an odd
    value of v makes the elements of o that see it odd, and no others' rows"""
    n, cut, D = 300, 40, 128
    q, k, v, do = (normal((n, h, D), 20 + i, type) for i, h in enumerate((2, 1, 1, 2)))
    how = dict(scale=0.1, window=50)
    ones = torch.ones(n)
    ref = au.batch(q, k, v, [0, n], [0, n], float(np.float32(0.1)), window=50, dout=torch.where((ones.cumsum(0) > cut)[:, None, None], do, torch.zeros((), dtype=type)))
    q[:cut, :, 5], do[:cut, :, 9] = float("nan"), float("inf")
    out, lse = f3m.attention(q.to(DEV), k.to(DEV), v.to(DEV), **how)
    dq, dk, dv = f3m.attention_grad(do.to(DEV), q.to(DEV), k.to(DEV), v.to(DEV), out, lse, **how)
    for y, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        au.close(y[cut:], {x: ref[x][cut:] for x in (name, name + "_tol")}, name)
    v[100, 0, 3] = float("nan")
    out, lse = f3m.attention(k.to(DEV), k.to(DEV), v.to(DEV), **how)
    out = out.float().cpu()
    assert torch.isnan(out[100:150, :, 3]).all() and torch.isfinite(out[:100]).all() and torch.isfinite(out[150:]).all()
    assert torch.isfinite(lse).all()


def test_offsets_that_lie():
    """offsets outside the tensors, or falling, are cut: no access leaves the tensors, good sequences of the batch are right"""
    n, D = 100, 64
    q = normal((n, 2, D), 1, BF)
    x = q.to(DEV)
    off = dev_offsets([0, 50, 40, 100000, -5])
    out, lse = f3m.attention(x, x, x, q_offsets=off, k_offsets=off, max_q=50, max_k=50, scale=0.125)
    dq, dk, dv = f3m.attention_grad(x, x, x, x, out, lse, q_offsets=off, k_offsets=off, max_q=50, max_k=50, scale=0.125)
    torch.cuda.synchronize()
    want = au.batch(q[:40], q[:40], q[:40], [0, 40], [0, 40], 0.125)
    au.close(out[:40], want, "out")


def test_gaussian_smoother_is_the_ratio_of_two_exact_products():
    """q = (x, 1, 1, 1)/gamma, k = (y, the three 8-bit pieces of -|y|^2/2)/gamma: the attention of v over all keys is the Gaussian smoother
    K(X,Y) v / K(X,Y) 1, which direct_kmvm_xy gives column by column"""
    nx, ny, gamma = 500, 700, 0.5
    X, Y = normal((nx, 3), 1, BF).float(), normal((ny, 3), 2, BF).float()
    v = normal((ny, 1, 8), 3, BF)
    rest, pieces = -(Y.double() ** 2).sum(1) / 2, []
    for _ in range(3):
        pieces.append(rest.to(BF))
        rest = rest - pieces[-1].double()
    q, k = torch.zeros((nx, 1, 8), dtype=BF), torch.zeros((ny, 1, 8), dtype=BF)
    q[:, 0, :3], q[:, 0, 3:6] = X.to(BF), 1.0
    k[:, 0, :3] = Y.to(BF)
    for i, x in enumerate(pieces):
        k[:, 0, 3 + i] = x
    out, lse = f3m.attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=1.0 / gamma ** 2, causal=False)
    Xd, Yd, vd = X.to(DEV).contiguous(), Y.to(DEV).contiguous(), v.to(DEV)
    one = f3m.direct_kmvm_xy(Xd, Yd, torch.ones(ny, device=DEV), gamma).double()
    for c in range(8):
        col = vd[:, 0, c].float().contiguous()
        want = f3m.direct_kmvm_xy(Xd, Yd, col, gamma).double() / one
        mass = f3m.direct_kmvm_xy(Xd, Yd, col.abs(), gamma).double() / one
        # bf16 has 8 significant bits, steps of 2^-7 at 1: a rounding is off by 2^-8 of the value at most.  Weights: sum_j 2^-8 w_j |v_j| = 2^-8
        # mass; the result: 2^-8 |o| <= 2^-8 mass (1 + 2^-8); together 2^-7 1.01 mass.  Products in fp32: exponents up to 40, 2^-24 each
        assert ((out[:, 0, c].double() - want).abs() <= 2.0 ** -7 * 1.02 * mass + 1e-4 * mass).all()
    # and its normaliser: log K(X,Y) 1 = lse - |x|^2 / (2 gamma^2)
    assert ((lse[:, 0].double() - (X.to(DEV).double() ** 2).sum(1) / (2 * gamma ** 2)) - one.log()).abs().max() < 1e-4


def test_gradient_against_differences():
    """sum(out * dout) and its central differences along random directions, in 64 bits of the definition: the formula's gradients; and the
    kernel's gradients along the same directions, whose error adds up over the elements"""
    n, D = 60, 32
    q, k, v, do = (normal((n, 2, D), 40 + i, BF) for i in range(4))
    how = dict(window=20, sinks=3)
    out, lse = f3m.attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=0.2, **how)
    grads = f3m.attention_grad(do.to(DEV), q.to(DEV), k.to(DEV), v.to(DEV), out, lse, scale=0.2, **how)
    scale = float(np.float32(0.2))
    want = au.batch(q, k, v, [0, n], [0, n], scale, dout=do, **how)

    def loss(x):
        return (au.batch(*x, [0, n], [0, n], scale, type=BF, **how)["out"] * do.double()).sum()

    for i, name in enumerate(("dq", "dk", "dv")):
        step = normal((n, 2, D), 50 + i, torch.float64)
        ends = []
        for sign in (1, -1):
            x = [q.double(), k.double(), v.double()]
            x[i] = x[i] + sign * 1e-4 * step
            ends.append(loss(x))
        slope = (ends[0] - ends[1]) / 2e-4
        assert abs(slope - (want[name] * step).sum()) < 1e-5 * (want[name] * step).abs().sum()
        assert abs(slope - (grads[i].cpu().double() * step).sum()) <= (want[name + "_tol"] * step.abs()).sum() + 1e-5 * (want[name] * step).abs().sum()


def test_same_bits_again():
    x = normal((700, 8, 128), 3, BF).to(DEV)
    k = normal((700, 2, 128), 4, BF).to(DEV)
    first = None
    for _ in range(3):
        out, lse = f3m.attention(x, k, k, window=300, sinks=4)
        got = (out, lse) + f3m.attention_grad(x, x, k, k, out, lse, window=300, sinks=4)
        if first is not None:
            assert all(torch.equal(a, b) for a, b in zip(first, got))
        first = got


def test_graph_replays_and_streams():
    """a training step's calls captured once: every replay computes what the inputs hold then; two graphs do not share workspace"""
    n = 300
    side = torch.cuda.Stream()
    x = torch.zeros((n, 4, 64), dtype=BF, device=DEV)
    k = torch.zeros((n, 2, 64), dtype=BF, device=DEV)
    one = torch.zeros((1, 4, 64), dtype=BF, device=DEV)
    graphs, results = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out, lse = f3m.attention(x, k, k, window=90, sinks=1)
            last = f3m.attention(one, k, k)      # in parts
            got = (out, lse) + f3m.attention_grad(x, x, k, k, out, lse, window=90, sinks=1) + last
        graphs.append(g)
        results.append(got)
    for seed in range(4):
        x.copy_(normal(x.shape, seed, BF))
        k.copy_(normal(k.shape, seed + 10, BF))
        one.copy_(normal(one.shape, seed + 20, BF))
        graphs[seed % 2].replay()
        graphs[1 - seed % 2].replay()
        out, lse = f3m.attention(x, k, k, window=90, sinks=1)
        want = (out, lse) + f3m.attention_grad(x, x, k, k, out, lse, window=90, sinks=1) + f3m.attention(one, k, k)
        torch.cuda.synchronize()
        for got in results:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    # a stream of the caller's that is not the current one
    torch.cuda.synchronize()
    out2, lse2 = f3m.attention(x, k, k, window=90, sinks=1, stream=side)
    grads = f3m.attention_grad(x, x, k, k, out2, lse2, window=90, sinks=1, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out2, lse2) + grads, want))


def test_empty_calls():
    q, k = torch.zeros((0, 4, 64), dtype=BF, device=DEV), normal((5, 2, 64), 1, BF).to(DEV)
    out, lse = f3m.attention(q, k, k)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    dq, dk, dv = f3m.attention_grad(q, q, k, k, out, lse)
    assert not dk.any() and not dv.any() and dq.shape == (0, 4, 64)
    out, lse = f3m.attention(k, k[:0], k[:0])
    assert not out.any() and (lse == -float("inf")).all()
    dq, dk, dv = f3m.attention_grad(k, k, k[:0], k[:0], out, lse)
    assert not dq.any() and dk.shape == (0, 2, 64)
    none = torch.zeros(1, dtype=torch.int32, device=DEV)
    f3m.attention(k, k, k, q_offsets=none, k_offsets=none)


def test_binding_refuses():
    x = torch.zeros((4, 2, 64), dtype=BF, device=DEV)
    with pytest.raises(TypeError):
        f3m.attention(x.float(), x, x)
    with pytest.raises(TypeError):
        f3m.attention(x[0], x, x)
    with pytest.raises(ValueError):
        f3m.attention(x, x.half(), x)
    with pytest.raises(ValueError):
        f3m.attention(x, x, x[:3])
    with pytest.raises(ValueError):
        f3m.attention(x, x, x, q_offsets=torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(TypeError):
        f3m.attention(x, x, x, q_offsets=torch.zeros(2, dtype=torch.int64, device=DEV), k_offsets=torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        f3m.attention(x[:, :, ::2], x[:, :, ::2], x[:, :, ::2])
    y = torch.zeros(4 * 2 * 64 + 8, dtype=BF, device=DEV)
    with pytest.raises(ValueError):
        f3m.attention(y[4:4 + 512].view(4, 2, 64), x, x)
    with pytest.raises(f3m.F3MError):
        f3m.attention(x, x, x, out=torch.zeros((4, 1, 64), dtype=BF, device=DEV).expand(4, 2, 64))
    with pytest.raises(f3m.F3MError):
        f3m.attention(x, x, x, window=5, causal=False)
    with pytest.raises(TypeError):
        f3m.attention_grad(x, x, x, x, x, None)
    with pytest.raises(f3m.F3MError) as e:
        f3m.attention(torch.zeros((4, 2, 136), dtype=BF, device=DEV), *[torch.zeros((4, 2, 136), dtype=BF, device=DEV)] * 2)
    assert e.value.status == 3


@pytest.mark.parametrize("sinks", [300, 2 ** 31 - 64, 2 ** 31 - 1])
def test_sinks_past_the_sequence(sinks):
    run(BF, 32, 2, 2, [300, 3], window=7, sinks=sinks)
    run(BF, 32, 2, 1, [3], [300], window=7, sinks=sinks)


@pytest.mark.parametrize("type", [BF, HF])
@pytest.mark.parametrize("D,Hq,Hk,nq,nk,how", [(64, 1, 1, [1900], None, {}), (128, 3, 1, [1400, 1, 650], None, {}), (80, 2, 2, [1300], [1450], {}),
                                               (40, 2, 1, [1700, 90], None, dict(window=1200, sinks=3)), (128, 1, 1, [1600], None, dict(window=150, sinks=200)),
                                               (128, 2, 1, [45], [1800], {}), (64, 1, 1, [130, 0], [1500, 70], dict(causal=False))])
def test_gradients_of_long_sequences_and_few_heads(type, D, Hq, Hk, nq, nk, how):
    """few tiles of rows and keys: both are cut into parts, whose sums are added up"""
    run(type, D, Hq, Hk, nq, nk, seed=D + len(nq), **how)


def test_gradients_in_parts_past_the_given_maxima():
    """tokens past max_q and keys past max_k are left out of the gradients, the rest is as without them; again gives the same bits"""
    n, D = 1500, 64
    q, k, v, do = (normal((n, 1, D), 60 + i, BF).to(DEV) for i in range(4))
    off = dev_offsets([0, n])
    out, lse = f3m.attention(q, k, v)
    whole = f3m.attention_grad(do, q, k, v, out, lse)
    grads = [torch.full_like(q, 7.0) for _ in range(3)]
    for _ in range(2):
        got = f3m.attention_grad(do, q, k, v, out, lse, q_offsets=off, k_offsets=off, max_q=n, max_k=640, dq=grads[0], dk=grads[1], dv=grads[2])
        assert all((x[640:] == 7.0).all() for x in got[1:])
        for x, y in zip(got, whole):      # sums in other parts: in fp32, so no more than a step of bf16 apart, 2^-7 of a value
            z = torch.where(x == 7.0, y, x).float() - y.float()
            assert (z.abs() <= 2.0 ** -7 * y.float().abs() + 2.0 ** -12).all()
    again = f3m.attention_grad(do, q, k, v, out, lse)
    assert all(torch.equal(x, y) for x, y in zip(again, whole))
    for x in grads:
        x.fill_(7.0)
    f3m.attention_grad(do, q, k, v, out, lse, q_offsets=off, k_offsets=off, max_q=300, max_k=n, dq=grads[0], dk=grads[1], dv=grads[2])
    assert (grads[0][300:] == 7.0).all() and not (grads[0][:300] == 7.0).all(-1).any()
