"""Attention in 64 bits, one sequence and head at a time, from the definition; with it, for every result, how far a kernel may be off that
rounds where the library says it rounds: weights and their gradients to the type before the products, results at the end
(half a step u = finfo.eps / 2 each), everything else in fp32.

fp32 part: a score is a sum of D <= 128 products, off by no more than D 2^-24 times the sum of their sizes, in practice about
sqrt(D) 2^-24 of it, 1e-6 to 4e-6 here; exp2 and the sums add about as much.  2^-16 = 1.5e-5 of the sum of sizes covers them.
"""
import torch

FP32 = 2.0 ** -16


def visible(nq, nk, causal, window, sinks):
    pos = torch.arange(nq)[:, None] + (nk - nq)
    j = torch.arange(nk)[None, :]
    if not causal:
        return torch.ones((nq, nk), dtype=torch.bool)
    seen = j <= pos
    if window:
        seen &= (j > pos - window) | (j < sinks)
    return seen


def sequence(q, k, v, seen, scale, u, narrow, dout=None):
    """one head: q (nq, D), k, v (nk, D) fp64 -> dict of results and tolerances; hidden entries may hold anything"""
    s = torch.where(seen, q @ k.T * scale, torch.full((), -torch.inf, dtype=torch.float64))
    lse = torch.logsumexp(s, -1) if k.shape[0] else torch.full((q.shape[0],), -torch.inf, dtype=torch.float64)
    none = torch.isinf(lse) & (lse < 0)
    p = torch.where(seen & ~none[:, None], torch.exp(s - torch.where(none, 0.0, lse)[:, None]), torch.zeros((), dtype=torch.float64))
    o, mass = p @ v, p @ v.abs()
    got = {"out": o, "lse": lse, "out_tol": u * (mass + o.abs()) * 1.01 + FP32 * mass + (2.0 ** -32 * v.abs().sum(0) if narrow else 0.0) + 1e-30,
           "lse_tol": FP32 * (1 + torch.where(none, 0.0, lse).abs() + scale * (q.abs() @ k.abs().T).amax(-1) if k.shape[0] else torch.ones_like(lse))}
    if narrow:      # a result below fp16's normal range is rounded to steps of 2^-24
        got["out_tol"] = got["out_tol"] + 2.0 ** -25
    if dout is not None:
        dp = dout @ v.T
        ds = p * (dp - (dout * o).sum(-1, keepdim=True))
        size = p * (dout.abs() @ v.abs().T + (dout.abs() * mass).sum(-1, keepdim=True))
        # dS: its own rounding, out's rounding inside dO.out, fp32
        tol = u * ds.abs() * 1.01 + u * p * (dout.abs() * o.abs()).sum(-1, keepdim=True) + FP32 * size
        tp = u * p * 1.01 + FP32 * p
        if narrow:
            tol = tol + 2.0 ** -38 * (ds.abs().amax() if ds.numel() else 0.0) + p * 2.0 ** -25 * dout.abs().sum(-1, keepdim=True)
            tp = tp + 2.0 ** -36
        end = 2.0 ** -25 if narrow else 1e-30
        dq, dk, dv = ds @ k * scale, ds.T @ q * scale, p.T @ dout
        got.update(dq=dq, dk=dk, dv=dv, dq_tol=tol @ k.abs() * scale + u * dq.abs() * 1.01 + end, dk_tol=tol.T @ q.abs() * scale, dv_tol=tp.T @ dout.abs(),
                   end=end)
    return got


def batch(q, k, v, q_off, k_off, scale, causal=True, window=0, sinks=0, dout=None, type=None):
    """packed tensors (CPU, any type) -> dict of fp64 results and tolerances in the same layout; rows of no sequence are NaN"""
    type = type or q.dtype
    u, narrow = torch.finfo(type).eps / 2, type == torch.float16
    q64, k64, v64 = q.double(), k.double(), v.double()
    d64 = None if dout is None else dout.double()
    g = q.shape[1] // k.shape[1]
    nan = lambda x: torch.full(x.shape, torch.nan, dtype=torch.float64)   # noqa: E731
    r = {"out": nan(q), "out_tol": nan(q), "lse": nan(q[..., 0]), "lse_tol": nan(q[..., 0])}
    if dout is not None:
        r.update({n: nan(q) for n in ("dq", "dq_tol")})
        r.update({n: nan(k) for n in ("dk", "dk_tol", "dv", "dv_tol")})
    for b in range(len(q_off) - 1):
        a, e, c, f = q_off[b], q_off[b + 1], k_off[b], k_off[b + 1]
        seen = visible(e - a, f - c, causal, window, sinks)
        if dout is not None:
            for n in ("dk", "dk_tol", "dv", "dv_tol"):
                r[n][c:f] = 0.0
        for h in range(q.shape[1]):
            x = sequence(q64[a:e, h], k64[c:f, h // g], v64[c:f, h // g], seen, scale, u, narrow, None if dout is None else d64[a:e, h])
            for n in ("out", "out_tol", "lse", "lse_tol") + (("dq", "dq_tol") if dout is not None else ()):
                r[n][a:e, h] = x[n]
            if dout is not None:
                for n in ("dk", "dk_tol", "dv", "dv_tol"):
                    r[n][c:f, h // g] += x[n]
    if dout is not None:
        for n in ("dk", "dv"):
            r[n + "_tol"] += u * r[n].abs() * 1.01 + (2.0 ** -25 if narrow else 1e-30)
    return r


def close(got, want, name):
    """asserts |got - want| <= tol wherever want is a number, and the same infinities"""
    x, y, t = got.detach().cpu().double(), want[name], want[name + "_tol"]
    some = ~torch.isnan(y)
    inf = torch.isinf(y) & some
    assert torch.equal(x[inf], y[inf]), "%s: infinities differ" % name
    some &= ~inf
    off = (x - y).abs()[some]
    assert not torch.isnan(off).any(), "%s: NaN" % name
    over = off - t[some]
    if off.numel():
        assert over.max() <= 0, "%s: off by %.3g, %.3g allowed (%d of %d over)" % (name, off[over.argmax()], t[some][over.argmax()], int((over > 0).sum()), off.numel())


def offsets(lengths):
    o = [0]
    for n in lengths:
        o.append(o[-1] + n)
    return o
