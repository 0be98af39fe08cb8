"""The cases on which the serving and training operators around the quantized linear layer are measured.

Four operators of a block with 4-bit weights, 8-bit activations and an 8-bit cache:

  norm_fwd  residual addition, root-mean-square norm and per-token 8-bit quantization of the result
  norm_bwd  its gradient (straight through the quantizer)
  kv        new keys and values quantized into a paged 8-bit cache (one scale per block of tokens and
            head), and the blocks they touched read back
  attn      causal grouped-query attention of the newest tokens of each sequence over such a cache

`run` is the operators' plain form in elementary torch operations where `own` is false, and the calls
into this package where it is true.
"""
import math
import random

import torch

own = False

EPS = 1e-5
INF = float("inf")


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of a 4096-wide model enters a block: the latency of a decode step
        dict(name="norm_fwd_token", op="norm_fwd", T=1, k=4096, residual=True, out="x_hat"),
        # the token batch of the 13B layer workload, X_hat straight into the quantized linears
        dict(name="norm_fwd_layer", op="norm_fwd", T=16384, k=5120, residual=True, out="x_hat"),
        # a training forward that keeps its activations as 8-bit codes and rebuilds X_hat from them;
        # an odd micro-batch
        dict(name="norm_fwd_codes", op="norm_fwd", T=8191, k=4096, residual=True, out="codes"),
        # the backward of a small, odd micro-batch
        dict(name="norm_bwd_small", op="norm_bwd", T=333, k=4096, residual=True),
        # the backward at the 13B layer workload's token batch
        dict(name="norm_bwd_layer", op="norm_bwd", T=16384, k=5120, residual=True),
        # one decode step appends a token to each of 48 ragged sequences, two of them idle slots
        dict(name="kv_token", op="kv", seqs=48, heads_kv=8, d=128, block=16, new=1, hist=4000, idle=2, ragged=3),
        # ragged prompts of a model with 40 full heads enter the cache, some behind a cached prefix
        dict(name="kv_prompt", op="kv", seqs=9, heads_kv=40, d=128, block=64, new=4001, hist=77, idle=0, ragged=5),
        # one sequence, one token, a short conversation: latency
        dict(name="attn_one", op="attn", seqs=1, heads=32, heads_kv=8, d=128, block=16, new=1, hist=1029, window=0,
             idle=0, ragged=0),
        # a serving step of 64 ragged sequences, three of them idle slots
        dict(name="attn_batch", op="attn", seqs=64, heads=32, heads_kv=8, d=128, block=64, new=1, hist=8100, window=0,
             idle=3, ragged=7),
        # two very long sequences: few rows, a long axis
        dict(name="attn_long", op="attn", seqs=2, heads=32, heads_kv=8, d=128, block=32, new=1, hist=131001, window=0,
             idle=0, ragged=0),
        # a few drafted tokens per sequence verified at once, full heads, sliding window
        dict(name="attn_draft", op="attn", seqs=16, heads=40, heads_kv=40, d=128, block=16, new=5, hist=2500,
             window=2048, idle=0, ragged=9),
        # ragged prompts behind cached prefixes: compute-bound
        dict(name="attn_prompt", op="attn", seqs=4, heads=32, heads_kv=8, d=128, block=64, new=4000, hist=500,
             window=0, idle=0, ragged=11),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "kv", "attn_token", "attn_draft", "attn_prompt"])
    if op.startswith("norm"):
        k = 8 * _log(rng, 32, 1792)
        k += 8 if k == 3 * 1024 else 0
        T = _log(rng, 1, max(1, min(16384, 16384 * 5120 // k)))
        T += T == 3 * 1024
        c = dict(op=op, T=T, k=k, residual=rng.random() < 0.8)
        if op == "norm_fwd":
            c["out"] = rng.choice(["x_hat", "codes", "bf16"])
        return c
    heads_kv, group = rng.choice([(8, 4), (32, 1), (40, 1), (8, 8), (1, 16), (4, 7)])
    c = dict(op="kv" if op == "kv" else "attn", heads_kv=heads_kv, d=rng.choice([64, 128, 128]),
             block=rng.choice([16, 32, 64, 128]), idle=0, ragged=rng.randrange(1, 1 << 20))
    if op == "kv":
        c["new"] = _log(rng, 1, 4001)
        c["hist"] = rng.choice([0, _log(rng, 1, 4000)])
        c["seqs"] = _log(rng, 1, max(1, min(64, 9 * 4001 * 40 // (heads_kv * (c["new"] + c["hist"])))))
    else:
        c["heads"] = heads_kv * group
        c["window"] = rng.choice([0, 0, 0, _log(rng, 1, 4096)])
        if op == "attn_prompt":
            # at most the listed prompt's scores
            c["new"] = _log(rng, 33, 4000)
            c["hist"] = rng.choice([0, _log(rng, 1, 4000)])
            room = 4 * 4000 * 4500 * 32 // (c["heads"] * c["new"] * (c["new"] + c["hist"]))
        else:
            c["new"] = 1 if op == "attn_token" else _log(rng, 2, 32)
            c["hist"] = _log(rng, 1, 131001)
            room = 2 * 131001 * 8 // (heads_kv * (c["new"] + c["hist"]))
        if room < 1:
            c["hist"] = c["hist"] // 64
            room = 1
        c["seqs"] = _log(rng, 1, max(1, min(64, room)))
        if c["seqs"] > 2 and c["new"] == 1:
            c["idle"] = rng.choice([0, 1])
    for f in ("new", "hist", "window"):
        c[f] = c.get(f, 0) + (c.get(f, 0) == 3 * 1024)
    return c


def lengths(case):
    """Per sequence (tokens in the cache with the new ones, new tokens); the last `idle` slots hold no sequence,
    so their one row is at no position."""
    rng = random.Random(case["ragged"])
    new, hist = case["new"], case["hist"]
    out = []
    for b in range(case["seqs"]):
        if b >= case["seqs"] - case["idle"]:
            out.append((0, 1))
        elif b == 0 or not case["ragged"]:
            out.append((hist + new, new))
        else:
            n = rng.randint((new + 1) // 2, new)
            out.append((rng.randint(0, hist) + n, n))
    return out


def pairs(case):
    """Pairs (query, key) that the mask of `attn` leaves, over all sequences, and the keys that any query sees."""
    w, total, keys = case["window"], 0, 0
    for length, n in lengths(case):
        if length == 0:
            continue
        first, last = length - n, length - 1
        if w:
            full = max(0, last - max(first, w - 1) + 1)            # positions that see w keys
            part = [p + 1 for p in (first, min(last, w - 2))] if first <= w - 2 else None
            total += full * w + ((part[0] + part[1]) * (part[1] - part[0] + 1) // 2 if part else 0)
            keys += length - max(0, first - w + 1)
        else:
            total += (first + 1 + last + 1) * n // 2
            keys += length
    return total, keys


def work(case):
    op = case["op"]
    if op == "norm_fwd":
        n = case["T"] * case["k"]
        # X (and R) in; H out where there is a residual; the values out; with "codes" the codes out and in again
        b = n * (2 + 2 + (4 if case["residual"] else 0) + (2 if case["out"] == "codes" else 0)) + 2 * case["k"]
        b += 0 if case["out"] == "bf16" else 4 * case["T"]
        return {"bytes": b, "flops": 10 * n}
    if op == "norm_bwd":
        n = case["T"] * case["k"]
        return {"bytes": n * (6 + (2 if case["residual"] else 0)) + 6 * case["k"], "flops": 14 * n}
    d, hkv, P = case["d"], case["heads_kv"], case["block"]
    if op == "kv":
        new = sum(n for length, n in lengths(case) if length)
        back = sum(length - (length - n) // P * P for length, n in lengths(case) if length)
        # K and V: bf16 in, 8 bits out, 8 bits in, bf16 out
        return {"bytes": 2 * hkv * d * (3 * new + 3 * back), "flops": 2 * hkv * d * (4 * new + back)}
    rows = sum(n for _, n in lengths(case))
    seen, keys = pairs(case)
    scales = sum(-(-length // P) for length, _ in lengths(case)) * hkv * 8
    return {"bytes": 2 * keys * hkv * d + scales + 4 * rows * case["heads"] * d,
            "flops": 4 * seen * case["heads"] * d}


# ---------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    st = dict(case)
    if case["op"].startswith("norm"):
        T, k = case["T"], case["k"]
        # hidden states have a few channels that are much larger than the others
        channel = torch.where(torch.rand(k, generator=g, device="cuda") < 4e-3, 12.0, 1.0)
        st["gamma"] = (1.0 + 0.2 * normal(k)).bfloat16()
        st["X"] = (normal(T, k) * 0.3).bfloat16()
        st["R"] = (normal(T, k) * channel).bfloat16() if case["residual"] else None
        if case["op"] == "norm_bwd":
            st["H"] = (normal(T, k) * channel).bfloat16()
            st["dY"] = normal(T, k).bfloat16()
            st["dH"] = normal(T, k).bfloat16() if case["residual"] else None
            del st["X"], st["R"]
        return st
    hkv, d, P = case["heads_kv"], case["d"], case["block"]
    ls = lengths(case)
    blocks = [-(-length // P) for length, _ in ls]
    width = max(1, max(blocks))
    pool = sum(blocks) + 3
    order = torch.randperm(pool, generator=g, device="cuda").int()
    at, tables = 0, torch.zeros(case["seqs"], width, dtype=torch.int32, device="cuda")
    for b, n in enumerate(blocks):
        tables[b, :n] = order[at:at + n]
        at += n
    st["table"] = tables
    st["rows"] = sum(n for _, n in ls)
    st["max_new"] = max(n for _, n in ls)
    st["max_len"] = max(length for length, _ in ls)
    start = [0]
    for _, n in ls:
        start.append(start[-1] + n)
    st["lens"] = torch.tensor([length for length, _ in ls], dtype=torch.int32, device="cuda")
    st["start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
    # a block's largest magnitude is its scale times 127; keys have a few large channels
    for name in ("k", "v"):
        codes = normal(pool, hkv, P, d)
        if name == "k":
            codes *= torch.where(torch.rand(hkv, 1, d, generator=g, device="cuda") < 0.03, 4.0, 1.0)
        amax = codes.abs().amax((2, 3))
        st[name + "_codes"] = (codes * (127.0 / amax)[:, :, None, None]).round().to(torch.int8)
        st[name + "_scale"] = amax / 127.0
    if case["op"] == "kv":
        # new keys and values as two parts of one projection's output, a little larger here and there
        kv = normal(st["rows"], 2, hkv, d)
        kv *= torch.where(torch.rand(st["rows"], 2, hkv, 1, generator=g, device="cuda") < 0.2, 1.5, 1.0)
        kv = kv.bfloat16()
        st["K"], st["V"] = kv[:, 0], kv[:, 1]
        # the blocks that the new tokens touch, read back from their first token on
        back = [length - max(0, length - n) // P * P for length, n in ls]
        st["back_rows"], st["back_max"] = sum(back), max(back)
        starts = [0]
        for n in back:
            starts.append(starts[-1] + n)
        st["back_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    else:
        # queries as the first part of a projection's output that also holds keys and values
        qkv = normal(st["rows"], case["heads"] + 2 * hkv, d).bfloat16()
        st["Q"] = qkv[:, :case["heads"]]
        st["scale"] = 1.5 / math.sqrt(d)
    return st


# ---------------------------------------------------------------------------- the plain forms
def _norm_fwd(st):
    x = st["X"].float()
    h = x + st["R"].float() if st["residual"] else x
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * st["gamma"].float()
    out = [h.bfloat16()] if st["residual"] else []
    if st["out"] == "bf16":
        return out + [y.bfloat16()]
    amax = y.abs().amax(1, keepdim=True)
    s = torch.where(amax > 0, amax / 127.0, torch.ones_like(amax))
    return out + [(torch.clamp(torch.round(y / s), -128, 127) * s).bfloat16(), s[:, 0]]


def _norm_bwd(st):
    h, dy, gamma = st["H"].float(), st["dY"].float(), st["gamma"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    g = dy * gamma
    dx = r * (g - h * (r * r * (g * h).mean(1, keepdim=True)))
    if st["residual"]:
        dx = dx + st["dH"].float()
    return [dx.bfloat16(), (dy * h * r).sum(0)]


def _places(lens, start, rows):
    """Sequence, row within it and position in it of each of `rows` rows (the newest of each sequence)."""
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(start.long(), r, right=True) - 1
    i = r - start.long()[b]
    return b, i, lens.long()[b] - (start[1:] - start[:-1]).long()[b] + i


def _kv_write(codes, scale, new, st, at):
    """`new` [rows, heads, d] quantized into codes [blocks, heads, P, d], scale [blocks, heads]; `at` from _places."""
    P = st["block"]
    b, _, pos = at
    keep = pos >= 0
    new, b, pos = new[keep].float(), b[keep], pos[keep]
    blk, slot = st["table"].long()[b, pos // P], pos % P
    shape = scale.shape
    amax = torch.full(shape, -1.0, device="cuda").index_reduce_(0, blk, new.abs().amax(2), "amax")
    first = torch.full(shape[:1], P, device="cuda").scatter_reduce_(0, blk, slot, "amin")
    touched, old = amax >= 0, (first > 0)[:, None]
    fresh = torch.where(amax > 0, amax / 127.0, torch.ones_like(amax))
    s = torch.where(touched, torch.where(old, torch.maximum(scale, amax / 127.0), fresh), scale)
    # tokens that were in a block before move to its larger scale
    grown = (touched & old & (s > scale))[:, :, None, None] & (torch.arange(P, device="cuda") < first[:, None])[:, None, :, None]
    codes.copy_(torch.where(grown, torch.round(codes.float() * (scale / s)[:, :, None, None]), codes.float()))
    codes[blk, :, slot] = torch.clamp(torch.round(new / s[blk][:, :, None]), -127, 127).to(torch.int8)
    scale.copy_(s)


def _kv(st):
    at = _places(st["lens"], st["start"], st["rows"])
    _kv_write(st["k_codes"], st["k_scale"], st["K"], st, at)
    _kv_write(st["v_codes"], st["v_scale"], st["V"], st, at)
    b, _, pos = _places(st["lens"], st["back_start"], st["back_rows"])
    blk, slot = st["table"].long()[b, pos // st["block"]], pos % st["block"]
    return [(st[n + "_codes"][blk, :, slot].float() * st[n + "_scale"][blk][:, :, None]).bfloat16() for n in "kv"] + [
        st["k_scale"], st["v_scale"]]


def _attn(st):
    hkv, d, P, n = st["heads_kv"], st["d"], st["block"], st["max_new"]
    B, group = st["seqs"], st["heads"] // st["heads_kv"]
    table = st["table"].long()
    keys = table.shape[1] * P
    k, v = [(st[m + "_codes"][table].float() * st[m + "_scale"][table][..., None, None]).transpose(1, 2).reshape(
        B, hkv, keys, d) for m in "kv"]
    b, i, pos = _places(st["lens"], st["start"], st["rows"])
    q = torch.zeros(B, n, hkv, group, d, device="cuda")
    q[b, i] = st["Q"].float().reshape(-1, hkv, group, d)
    at = torch.full((B, n), -1, device="cuda")
    at[b, i] = pos
    j = torch.arange(keys, device="cuda")
    sees = (j <= at[:, :, None]) & ((j > at[:, :, None] - st["window"]) if st["window"] else True)
    s = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(B, hkv, n * group, d) * st["scale"], k.transpose(2, 3))
    s = torch.where(sees[:, None, :, None], s.view(B, hkv, n, group, keys), -INF)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -INF, m, torch.zeros_like(m)))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, hkv, n * group, keys), v).view(B, hkv, n, group, d) / torch.where(total > 0, total, 1.0)
    return [o.permute(0, 2, 1, 3, 4)[b, i].reshape(-1, st["heads"], d).bfloat16()]


# ---------------------------------------------------------------------------- the framework's operators
def _own(st):
    from paper_2406_06385_gb300 import lrqat as LQ
    new = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if st["op"].startswith("norm"):
        T, k = st["T"], st["k"]
        if st["op"] == "norm_bwd":
            norm = LQ.Norm(k, EPS, 8)
            dX, dgamma = new(T, k), new(k, dtype=torch.float32)
            ws = new(LQ.add_rmsnorm_bwd_workspace_bytes(norm, T), dtype=torch.uint8)
            LQ.add_rmsnorm_bwd(norm, T, st["dY"], st["dH"], st["H"], st["gamma"], dX, dgamma, False, ws)
            return [dX, dgamma]
        norm = LQ.Norm(k, EPS, 0 if st["out"] == "bf16" else 8)
        out = [new(T, k)] if st["residual"] else []
        H = out[0] if out else None
        Y = new(T, k)
        if st["out"] == "bf16":
            LQ.add_rmsnorm_fwd(norm, T, st["X"], st["R"], st["gamma"], H, Y, None, None)
            return out + [Y]
        s = new(T, dtype=torch.float32)
        if st["out"] == "x_hat":
            LQ.add_rmsnorm_fwd(norm, T, st["X"], st["R"], st["gamma"], H, Y, None, s)
        else:
            codes = new(T, k, dtype=torch.int8)
            LQ.add_rmsnorm_fwd(norm, T, st["X"], st["R"], st["gamma"], H, None, codes, s)
            LQ.act_dequant(norm, T, codes, s, Y)
        return out + [Y, s]
    cache = LQ.KVCache.of(st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"])
    batch = LQ.KVBatch.of(st["lens"], st["start"], st["table"], st["rows"], st["max_new"], st["max_len"])
    if st["op"] == "kv":
        LQ.kv_write(cache, batch, st["K"], st["V"])
        back = LQ.KVBatch.of(st["lens"], st["back_start"], st["table"], st["back_rows"], st["back_max"], st["max_len"])
        K, V = new(st["back_rows"], st["heads_kv"], st["d"]), new(st["back_rows"], st["heads_kv"], st["d"])
        LQ.kv_read(cache, back, K, V)
        return [K, V, st["k_scale"], st["v_scale"]]
    O = new(st["rows"], st["heads"], st["d"])
    ws = new(LQ.kv_attn_workspace_bytes(cache, batch, st["heads"], st["window"]), dtype=torch.uint8)
    LQ.kv_attn(cache, batch, st["Q"], st["scale"], st["window"], O, ws)
    return [O]


def run(state):
    if own:
        return _own(state)
    return {"norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd, "kv": _kv, "attn": _attn}[state["op"]](state)


# ---------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    D = torch.float64
    if case["op"] == "norm_fwd":
        h = st["X"].to(D)
        if case["residual"]:
            h += st["R"].to(D)
        out = [h] if case["residual"] else []
        y = h / torch.sqrt(torch.linalg.vecdot(h, h)[:, None] / case["k"] + EPS) * st["gamma"].to(D)
        if case["out"] == "bf16":
            return out + [y]
        s = torch.maximum(y.max(1).values, -y.min(1).values) / 127
        s[s == 0] = 1.0
        return out + [torch.round(y / s[:, None]).clamp(-128, 127) * s[:, None], s]
    if case["op"] == "norm_bwd":
        h, dy, gamma = st["H"].to(D), st["dY"].to(D), st["gamma"].to(D)
        rms = torch.sqrt(torch.linalg.vecdot(h, h)[:, None] / case["k"] + EPS)
        n = h / rms                                                # the normed row; y = n * gamma
        g = dy * gamma
        dx = (g - n * torch.linalg.vecdot(g, n)[:, None] / case["k"]) / rms
        return [dx + st["dH"].to(D) if case["residual"] else dx, torch.einsum("tk,tk->k", dy, n)]
    P, hkv, d = case["block"], case["heads_kv"], case["d"]
    table, start = st["table"].tolist(), st["start"].tolist()
    if case["op"] == "kv":
        back = ([], [])
        scales = (st["k_scale"].to(D), st["v_scale"].to(D))
        for b, (length, n) in enumerate(lengths(case)):
            if length == 0:
                continue
            for p0 in range((length - n) // P * P, length, P):
                blk, p1 = table[b][p0 // P], min(length, p0 + P)
                old = max(0, length - n - p0)
                rows = slice(start[b] + p0 + old - (length - n), start[b] + p1 - (length - n))
                for i, name in enumerate(("k", "v")):
                    x = st[name.upper()][rows].to(D)
                    s = x.abs().amax((0, 2)).div(127).float().to(D)    # scales are held in 32 bits
                    c = st[name + "_codes"][blk, :, :old].to(D)
                    if old:
                        was = scales[i][blk].clone()
                        s = torch.maximum(s, was)
                        c = torch.round(c * (was / s)[:, None, None])
                    s = torch.where(s > 0, s, 1.0)
                    c = torch.cat([c.transpose(0, 1), torch.round(x / s[:, None])])
                    back[i].append(c * s[:, None])
                    scales[i][blk] = s
        return [torch.cat(back[0]), torch.cat(back[1]), scales[0], scales[1]]
    group = case["heads"] // hkv
    out = torch.zeros(st["rows"], hkv, group, d, dtype=D, device="cuda")
    q = st["Q"].to(D).view(st["rows"], hkv, group, d)
    for b, (length, n) in enumerate(lengths(case)):
        if length == 0:
            continue
        blocks = st["table"][b, :-(-length // P)].long()
        k, v = [(st[m + "_codes"][blocks].to(D) * st[m + "_scale"][blocks].to(D)[..., None, None]).permute(
            1, 0, 2, 3).reshape(hkv, -1, d)[:, :length] for m in "kv"]
        for i in range(0, n, 256):
            rows = slice(start[b] + i, start[b] + min(n, i + 256))
            pos = torch.arange(length - n + i, length - n + min(n, i + 256), device="cuda")
            far = pos[:, None] - torch.arange(length, device="cuda")
            hidden = (far < 0) | (far >= (case["window"] or length))
            s = torch.einsum("rhgd,hkd->hgrk", q[rows], k) * st["scale"]
            out[rows] = torch.einsum("hgrk,hkd->rhgd", torch.softmax(s.masked_fill(hidden, -INF), -1), v)
    return [out.view(st["rows"], -1, d)]
