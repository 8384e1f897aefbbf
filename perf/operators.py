"""The row-normalised products (attention) that this library is timed on, and their plain forms.

  attend    f3m.attention: o_i = sum_j w_ij v_j with w_ij = exp(scale q_i.k_j) / (its sum over the visible j), packed
            sequences, heads that share keys, causal order, a sliding window, a few first keys that stay visible
  gradient  f3m.attention_grad: the gradients of q, k and v
  store     KVCache.write, then KVCache.read: keys and values quantised to 8 bits as they go into a paged cache, read back
  cached    KVCache.attention: a chunk of new tokens (one token up to thousands) against the keys of a paged cache

A case is a dict of plain values.  Lengths of the sequences of a batch follow from "sequences", "longest" and "spread" (0: all
as long as the longest), so that a case says all sizes.  Inputs are normal values, as products of normalised activations are.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
PAIR_COST = 2 * 8192 * 8192 * 8       # score entries (query, key, head) of the largest listed case, what a drawn one may have


def _attend(op, sequences, longest, heads, kv_heads, dim, type="bf16", spread=0.0, causal=True, window=0, sinks=0, keys=0):
    return dict(op=op, sequences=sequences, longest=longest, spread=spread, keys=keys, heads=heads, kv_heads=kv_heads, dim=dim,
                type=type, causal=causal, window=window, sinks=sinks)


def _store(tokens, slots, kv_heads, dim, type="bf16", page=16):
    return dict(op="store", tokens=tokens, slots=slots, kv_heads=kv_heads, dim=dim, type=type, page=page)


def _cached(sequences, new, longest, heads, kv_heads, dim, type="bf16", held="e4m3", spread=0.0, window=0, sinks=0, page=16):
    return dict(op="cached", sequences=sequences, new=new, longest=longest, spread=spread, heads=heads, kv_heads=kv_heads, dim=dim,
                type=type, held=held, window=window, sinks=sinks, page=page)


def listed():
    return [
        # a few short sequences of different lengths, where the latency of the call counts
        dict(_attend("attend", 3, 129, 4, 2, 64, type="fp16", spread=0.9), name="attend short ragged"),
        # documents of uneven length in one batch, a window of a thousand tokens and four first ones
        dict(_attend("attend", 4, 4099, 16, 4, 128, spread=0.8, window=1024, sinks=4), name="attend windowed ragged"),
        # one long text, every token before a token visible to it
        dict(_attend("attend", 1, 16384, 8, 8, 128), name="attend long causal"),
        # a smoother: targets against another set of sources, no order, many weights per source
        dict(_attend("attend", 1, 10007, 4, 4, 64, type="fp16", causal=False, keys=20000), name="attend smoother"),
        # the smallest training step: uneven short sequences, a head dimension that fills no tile
        dict(_attend("gradient", 3, 200, 6, 2, 80, type="fp16", spread=0.7), name="gradient short ragged"),
        # an ordinary training step: four sequences of two thousand tokens, four query heads to a key head
        dict(_attend("gradient", 4, 2048, 16, 4, 128), name="gradient 4 x 2048"),
        # a long text with a window and first tokens, small heads
        dict(_attend("gradient", 1, 8192, 16, 4, 64, window=1024, sinks=4), name="gradient windowed 8192"),
        # one step of a batch of sixty-four sequences, a token each
        dict(_store(64, 65536, 8, 128), name="store a step's 64 tokens"),
        # the prompt of a long text in one piece
        dict(_store(32768, 131072, 8, 128), name="store a prompt of 32768"),
        # one step of a batch: sixty-four sequences of up to eight thousand tokens, 8-bit cache
        dict(_cached(64, 1, 8192, 32, 8, 128, spread=0.9), name="cached step of 64"),
        # one token after a very long text, cache in 16 bits: the work has to be split along the keys
        dict(_cached(1, 1, 131072, 32, 8, 128, held="bf16"), name="cached token after 131072"),
        # a chunk of a long prompt after what came before it, 8-bit cache, window and first tokens
        dict(_cached(2, 1021, 16384, 32, 8, 128, spread=0.3, window=4096, sinks=4), name="cached chunk of 1021"),
    ]


def _log(rng, lo, hi):
    """a size from [lo, hi], spread over its logarithm"""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "gradient", "store", "cached"])
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8])
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 128])
    type = rng.choice(["bf16", "bf16", "fp16"])
    window = rng.choice([0, 0, _log(rng, 16, 4096)])
    sinks = rng.choice([0, 1, 4, 16]) if window else 0
    if op == "store":
        tokens = _log(rng, 1, 32768)
        return _store(tokens, 4 * max(1024, tokens), kv_heads, dim, type=type, page=rng.choice([8, 16, 32, 64, 128]))
    if op == "cached":
        new, sequences = rng.choice([1, 1, _log(rng, 2, 1024)]), _log(rng, 1, 64)
        longest = new + _log(rng, 1, 32768)
        while sequences * (longest + 8) * kv_heads * dim > 64 * 8192 * 8 * 128 or sequences * new * longest * kv_heads * group > PAIR_COST:
            longest, new = (longest + 1) // 2, max(1, min(new, (longest + 1) // 2) if new == 1 else new // 2)
        return _cached(sequences, min(new, longest), longest, kv_heads * group, kv_heads, dim, type=type, held=rng.choice([type, "e4m3", "e4m3"]),
                       spread=round(rng.uniform(0, 0.95), 2), window=window, sinks=sinks, page=rng.choice([8, 16, 32, 64, 128]))
    sequences, longest, causal = _log(rng, 1, 16), _log(rng, 16, 8192), rng.random() < 0.8
    keys = 0 if causal and rng.random() < 0.8 else _log(rng, 16, 8192)
    while sequences * longest * max(longest, keys) * kv_heads * group > PAIR_COST // (1 if op == "attend" else 4):
        longest, keys = (longest + 1) // 2, (keys + 1) // 2
    return _attend(op, sequences, longest, kv_heads * group, kv_heads, dim, type=type, spread=round(rng.uniform(0, 0.95), 2),
                   causal=causal, window=window if causal else 0, sinks=sinks if causal else 0, keys=keys)


def lengths(count, longest, spread):
    """`count` lengths from (1 - spread) longest up to longest, the first one the longest"""
    return [max(1, int(round(longest * (1.0 - spread * ((0.6180339887498949 * i) % 1.0))))) for i in range(count)]


def _sizes(case):
    """(queries, keys) of each sequence"""
    if case["op"] == "cached":
        keys = lengths(case["sequences"], case["longest"], case["spread"])
        return [min(case["new"], k) for k in keys], keys
    queries = lengths(case["sequences"], case["longest"], case["spread"])
    return queries, lengths(case["sequences"], case["keys"], case["spread"]) if case["keys"] else queries


def _pairs(case):
    """visible (query, key) pairs of one head"""
    total = 0
    for nq, nk in zip(*_sizes(case)):
        if not case.get("causal", True):
            total += nq * nk
            continue
        pos = torch.arange(nk - nq, nk, dtype=torch.int64)
        seen = (pos + 1).clamp(min=0)
        if case["window"]:
            low = (pos + 1 - case["window"]).clamp(min=0)                       # first key of the window
            seen = seen - low + torch.minimum(low, torch.tensor(case["sinks"]))
        total += int(seen.clamp(min=0).sum())
    return total


def _used_keys(case):
    """keys that some query sees, over all sequences"""
    total = 0
    for nq, nk in zip(*_sizes(case)):
        low = max(0, nk - nq + 1 - case["window"]) if case["window"] and case.get("causal", True) else 0
        total += nk - low + min(low, case["sinks"])
    return total


def work(case):
    hk, d = case["kv_heads"], case["dim"]
    if case["op"] == "store":       # 16-bit values in, codes and exponents written and read, 16-bit values out
        return {"bytes": case["tokens"] * (2 * hk * (2 * (2 * d) + 2 * (d + 1)) + 8), "flops": 0.0}
    hq, (queries, keys) = case["heads"], _sizes(case)
    tq, tk, pairs = sum(queries), sum(keys), _pairs(case) * case["heads"]
    if case["op"] == "attend":
        return {"bytes": 2 * d * (2 * tq * hq + 2 * tk * hk) + 4 * tq * hq, "flops": 4.0 * d * pairs}
    if case["op"] == "gradient":    # q, k, v, out, dout and the normalisers in, three gradients out
        return {"bytes": 2 * d * (4 * tq * hq + 4 * tk * hk) + 4 * tq * hq, "flops": 10.0 * d * pairs}
    row = d + 1 if case["held"] == "e4m3" else 2 * d
    return {"bytes": 2 * hk * row * _used_keys(case) + 4 * d * tq * hq + 4 * tq * hq, "flops": 4.0 * d * pairs}


# ---- inputs ----

def _normal(gen, shape, type):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(type)


def _offsets(sizes):
    return torch.tensor([0] + sizes, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(DEV)


def _exponents(x):
    """the least e with max|x| <= 448 2^e over the last dimension, as the byte e + 127"""
    m, e = torch.frexp(x.abs().amax(-1))
    byte = e.int() - 9 + (m > 0.875).int() + 127
    return torch.where(m == 0, torch.full_like(byte, 127), byte.clamp(1, 254)).to(torch.uint8)


def _codes(x, byte):
    return (x * torch.exp2(127.0 - byte.float())[..., None]).to(torch.float8_e4m3fn)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    hk, d, type = case["kv_heads"], case["dim"], TYPES[case["type"]]
    state = dict(case, scale=1.0 / math.sqrt(d))
    if case["op"] == "store":
        pages = -(-case["slots"] // case["page"])
        state["slot"] = torch.randperm(case["slots"], generator=gen, device=DEV)[:case["tokens"]].contiguous()
        if case["tokens"] > 8:      # a padded batch: some tokens have no place
            state["slot"][7::61] = -1
        # values of uneven size from head to head, as keys have
        size = torch.exp2(torch.randn((hk, 1), generator=gen, device=DEV))
        state["new_k"] = (_normal(gen, (case["tokens"], hk, d), torch.float32) * size).to(type)
        state["new_v"] = _normal(gen, (case["tokens"], hk, d), type)
        for name in ("k", "v"):
            state[name] = torch.zeros((pages, hk, case["page"], d), device=DEV).to(torch.float8_e4m3fn)
            state[name + "_exp"] = torch.full((pages, hk, case["page"]), 127, dtype=torch.uint8, device=DEV)
        return state
    queries, keys = _sizes(case)
    state["max_q"], state["max_k"] = max(queries), max(keys)
    state["q_offsets"] = _offsets(queries)
    state["q"] = _normal(gen, (sum(queries), case["heads"], d), type)
    if case["op"] == "cached":
        page = case["page"]
        counts = [-(-n // page) for n in keys]
        pages = sum(counts) + 3
        order = torch.randperm(pages, generator=gen, device=DEV).int()
        table = torch.full((len(keys), max(counts)), -1, dtype=torch.int32, device=DEV)
        at = 0
        for i, c in enumerate(counts):
            table[i, :c] = order[at:at + c]
            at += c
        state["table"], state["lengths"] = table, torch.tensor(keys, dtype=torch.int32, device=DEV)
        for name in ("k", "v"):
            x = _normal(gen, (pages, hk, page, d), type)
            state[name], state[name + "_exp"] = x, None
            if case["held"] == "e4m3":
                byte = _exponents(x.float())
                state[name], state[name + "_exp"] = _codes(x.float(), byte), byte
        return state
    state["k_offsets"] = _offsets(keys)
    state["k"] = _normal(gen, (sum(keys), hk, d), type)
    state["v"] = _normal(gen, (sum(keys), hk, d), type)
    if case["op"] == "gradient":
        state["out"], state["lse"] = _plain_attend(state)
        state["dout"] = _normal(gen, (sum(queries), case["heads"], d), type)
    return state


# ---- the plain forms: elementary operations in 32 bits on padded batches ----

def _padded(x, offsets, most):
    """rows of packed sequences as (sequences, most, ...) with zeros behind each one's end"""
    at = offsets[:-1, None].long() + torch.arange(most, device=DEV)
    inside = at < offsets[1:, None]
    y = x[at.clamp(max=max(0, x.shape[0] - 1))].float()
    return torch.where(inside.view(*inside.shape, *[1] * (y.dim() - 2)), y, torch.zeros((), device=DEV)), inside


def _visible(state, nq, nk, max_q, max_k):
    """(sequences, 1, 1, max_q, max_k) truth values"""
    i, j = torch.arange(max_q, device=DEV)[None, :, None], torch.arange(max_k, device=DEV)[None, None, :]
    nq, nk = nq.long()[:, None, None], nk.long()[:, None, None]
    seen = (i < nq) & (j < nk)
    if state.get("causal", True):
        pos = i + (nk - nq)
        near = j > pos - state["window"] if state["window"] else j >= 0
        seen = seen & (j <= pos) & (near | (j < state["sinks"]))
    return seen[:, None, None]


def _weights(state, q, k, seen):
    """q (sequences, kv heads, group, rows, dim), k (sequences, kv heads, 1, dim, keys): the weights and the logarithms of their sums"""
    s = torch.matmul(q, k).mul_(state["scale"])
    s.masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    e = s.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    lse = torch.log(total) + top
    return e.div_(torch.where(total > 0, total, torch.ones_like(total))), lse[..., 0]


def _heads_first(x, kv_heads):
    """(sequences, rows, heads, dim) as (sequences, kv heads, group, rows, dim)"""
    b, n, h, d = x.shape
    return x.view(b, n, kv_heads, h // kv_heads, d).permute(0, 2, 3, 1, 4).contiguous()


def _packed(x, inside):
    """(sequences, kv heads, group, rows, ...) back to the packed rows"""
    x = x.permute(0, 3, 1, 2, *range(4, x.dim())).flatten(2, 3)
    return x[inside]


def _held(x, *at):
    """x[at] in 32 bits; 8-bit codes are moved as bytes"""
    return x.view(torch.uint8)[at].view(x.dtype).float() if x.dtype == torch.float8_e4m3fn else x[at].float()


def _plain_set(state):
    q, inside = _padded(state["q"], state["q_offsets"], state["max_q"])
    if state["op"] == "cached":
        nk = state["lengths"]
        j = torch.arange(state["max_k"], device=DEV)
        page = state["table"][:, j // state["page"]].long().clamp(min=0)
        held = []
        for name in ("k", "v"):
            x = _held(state[name], page, slice(None), j % state["page"])        # (sequences, keys, kv heads, dim)
            if state[name + "_exp"] is not None:
                x = x * torch.exp2(state[name + "_exp"][page, :, j % state["page"]].float() - 127.0)[..., None]
            held.append(x)
        k, v = held
    else:
        nk = state["k_offsets"].diff()
        k, v = (_padded(state[name], state["k_offsets"], state["max_k"])[0] for name in ("k", "v"))
    seen = _visible(state, state["q_offsets"].diff(), nk, state["max_q"], state["max_k"])
    return _heads_first(q, state["kv_heads"]), _heads_first(k, state["kv_heads"]), _heads_first(v, state["kv_heads"]), seen, inside


def _plain_attend(state):
    q, k, v, seen, inside = _plain_set(state)
    p, lse = _weights(state, q, k.transpose(-1, -2).contiguous(), seen)
    return _packed(torch.matmul(p, v), inside).to(state["q"].dtype), _packed(lse, inside)


def _plain_gradient(state):
    q, k, v, seen, inside = _plain_set(state)
    dout, _ = _padded(state["dout"], state["q_offsets"], state["max_q"])
    dout = _heads_first(dout, state["kv_heads"])
    p, _ = _weights(state, q, k.transpose(-1, -2).contiguous(), seen)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), dout).sum(2, keepdim=True)
    dp = torch.matmul(dout, v.transpose(-1, -2).contiguous())
    ds = dp.sub_((p * dp).sum(-1, keepdim=True)).mul_(p).mul_(state["scale"])
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q).sum(2, keepdim=True)
    _, has = _padded(state["k"], state["k_offsets"], state["max_k"])
    type = state["q"].dtype
    return _packed(dq, inside).to(type), _packed(dk, has).to(type), _packed(dv, has).to(type)


def _plain_store(state):
    slot, page = state["slot"], state["page"]
    some = slot >= 0
    at = slot[some]
    out = []
    for name in ("k", "v"):
        x = state["new_" + name][some].float()
        byte = _exponents(x)
        state[name].view(torch.uint8)[at // page, :, at % page] = _codes(x, byte).view(torch.uint8)
        state[name + "_exp"][at // page, :, at % page] = byte
        back = _held(state[name], at // page, slice(None), at % page) * torch.exp2(state[name + "_exp"][at // page, :, at % page].float() - 127.0)[..., None]
        y = torch.zeros_like(state["new_" + name])
        y[some] = back.to(y.dtype)
        out.append(y)
    return out


def run(state):
    if not own:
        if state["op"] == "store":
            k, v = _plain_store(state)
        elif state["op"] == "gradient":
            dq, dk, dv = _plain_gradient(state)
        else:
            out, lse = _plain_attend(state)
    else:
        from paper_2202_01085_amd import f3m
        if state["op"] in ("store", "cached"):
            cache = f3m.KVCache(state["k"], state["v"], state["k_exp"], state["v_exp"])
        if state["op"] == "store":
            cache.write(state["new_k"], state["new_v"], state["slot"])
            k, v = cache.read(state["slot"], dtype=state["new_k"].dtype)
        elif state["op"] == "cached":
            out, lse = cache.attention(state["q"], state["table"], state["lengths"], state["q_offsets"], max_q=state["max_q"],
                                       max_k=state["max_k"], scale=state["scale"], window=state["window"], sinks=state["sinks"])
        else:
            how = dict(q_offsets=state["q_offsets"], k_offsets=state["k_offsets"], max_q=state["max_q"], max_k=state["max_k"],
                       scale=state["scale"], causal=state["causal"], window=state["window"], sinks=state["sinks"])
            if state["op"] == "attend":
                out, lse = f3m.attention(state["q"], state["k"], state["v"], **how)
            else:
                dq, dk, dv = f3m.attention_grad(state["dout"], state["q"], state["k"], state["v"], state["out"], state["lse"], **how)
    if state["op"] == "store":      # the values that the cache stands for, its codes and its exponents
        return {"k": k, "v": v, "k_codes": state["k"], "v_codes": state["v"], "k_exp": state["k_exp"], "v_exp": state["v_exp"]}
    if state["op"] == "gradient":
        return {"dq": dq, "dk": dk, "dv": dv}
    return {"out": out, "lse": lse}


# ---- the definitions in 64 bits, a sequence and a head at a time ----

def _exact_eighth(x):
    """x (fp64) rounded to four significant bits, ties to even, steps of at least 2^-9"""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return torch.round(x / step) * step


def _exact_store(state):
    got = {}
    for name in ("k", "v"):
        x = state["new_" + name].double()
        top = x.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(top / 448.0).clamp(min=-126))
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1, torch.where((top <= 448.0 * torch.exp2(e - 1)) & (e > -126), e - 1, e))
        e = torch.where(top == 0, torch.zeros_like(e), e)
        code = _exact_eighth(x / torch.exp2(e))
        some = state["slot"] >= 0
        got[name] = torch.where(some[:, None, None], code * torch.exp2(e), torch.zeros_like(code))
        pages = state[name].double()
        flat = pages.permute(0, 2, 1, 3).reshape(-1, *pages.shape[1::2])
        flat[state["slot"][some]] = code[some]
        got[name + "_codes"] = flat.view(pages.shape[0], pages.shape[2], pages.shape[1], -1).permute(0, 2, 1, 3).contiguous()
        got[name + "_exp"] = None
    return got


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "store":
        return _exact_store(state)
    queries, keys = _sizes(case)
    group, hk = case["heads"] // case["kv_heads"], case["kv_heads"]
    q = state["q"].double()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    if case["op"] == "gradient":
        dout, k_all, v_all = (state[n].double() for n in ("dout", "k", "v"))
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k_all), torch.zeros_like(v_all)
    q0 = k0 = 0
    for b, (nq, nk) in enumerate(zip(queries, keys)):
        pos = torch.arange(nk - nq, nk, device=DEV)[:, None]
        j = torch.arange(nk, device=DEV)[None, :]
        hidden = torch.zeros((nq, nk), dtype=torch.bool, device=DEV)
        if case.get("causal", True):
            hidden = j > pos
            if case["window"]:
                hidden = hidden | ((j <= pos - case["window"]) & (j >= case["sinks"]))
        for h in range(hk):
            if case["op"] == "cached":
                at = state["table"][b, :-(-nk // case["page"])].long()
                k, v = (state[n][at, h].double() * (1.0 if state[n + "_exp"] is None else torch.exp2(state[n + "_exp"][at, h].double() - 127.0)[..., None])
                        for n in ("k", "v"))
                k, v = k.reshape(-1, case["dim"])[:nk], v.reshape(-1, case["dim"])[:nk]
            else:
                k, v = state["k"][k0:k0 + nk, h].double(), state["v"][k0:k0 + nk, h].double()
            for hq in range(h * group, (h + 1) * group):
                s = (q[q0:q0 + nq, hq] @ k.T * state["scale"]).masked_fill(hidden, -math.inf)
                total = torch.logsumexp(s, -1, keepdim=True)
                p = torch.where(hidden | ~torch.isfinite(total), torch.zeros_like(s), torch.exp(s - total))
                lse[q0:q0 + nq, hq] = total[:, 0]
                o = p @ v
                out[q0:q0 + nq, hq] = o
                if case["op"] == "gradient":
                    do = dout[q0:q0 + nq, hq]
                    ds = p * (do @ v.T - (do * o).sum(-1, keepdim=True)) * state["scale"]
                    dq[q0:q0 + nq, hq] = ds @ k
                    dk[k0:k0 + nk, h] += ds.T @ q[q0:q0 + nq, hq]
                    dv[k0:k0 + nk, h] += p.T @ do
        q0, k0 = q0 + nq, k0 + nk
    return {"dq": dq, "dk": dk, "dv": dv} if case["op"] == "gradient" else {"out": out, "lse": lse}
