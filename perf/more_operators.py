"""The cases on which the operators around the 8-bit cache that make up a serving step's attention are measured.

Four operators, next to the norm, the cache and its attention:

  plan     cache blocks for the new tokens of each sequence, taken from a free list on the device: row starts, block
           tables, positions and slots; and blocks of shortened sequences given back ("what": extend, truncate)
  rope     norms of each head's queries and keys and their rotation by position in one pass, and the gradient
  sinks    causal grouped-query attention over the cache through a sliding window and a few first tokens
  shared   causal attention of a batch whose sequences start with the same cached tokens

`run` is the operators' plain form in elementary torch operations where `own` is false, and the calls
into this package where it is true.
"""
import math
import random

import torch

own = False

EPS = 1e-6
INF = float("inf")


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # a decode step appends a token to each of 48 running sequences: latency
        dict(name="plan_token", op="plan", what="extend", seqs=48, new=1, hist=4000, block=16, pinned=0, pad=3, ragged=2),
        # a burst of ragged prompts behind a pinned prefix gets its blocks
        dict(name="plan_prompt", op="plan", what="extend", seqs=900, new=701, hist=2500, block=16, pinned=20, pad=5,
             ragged=3),
        # a scheduler takes back rejected drafts and finished sequences of a large batch
        dict(name="plan_free", op="plan", what="truncate", seqs=2500, new=333, hist=900, block=32, pinned=0, pad=0,
             ragged=4),
        # the new tokens of a decode step, far positions, heads with norms
        dict(name="rope_token", op="rope", bwd=False, T=48, heads=32, heads_kv=8, d=128, rot=128, interleaved=False,
             norm=True, base=500000.0, far=131001, run=1),
        # the token batch of the 13B layer workload, 40 full heads without norms
        dict(name="rope_layer", op="rope", bwd=False, T=16384, heads=40, heads_kv=40, d=128, rot=128, interleaved=False,
             norm=False, base=10000.0, far=0, run=2048),
        # the backward of an odd micro-batch of packed sequences, grouped heads with norms
        dict(name="rope_bwd", op="rope", bwd=True, T=8191, heads=32, heads_kv=8, d=128, rot=128, interleaved=False,
             norm=True, base=500000.0, far=0, run=1777),
        # a decode step of 64 ragged sequences, three of them idle slots, long streams behind a window of 2000
        dict(name="sinks_batch", op="sinks", seqs=64, heads=32, heads_kv=8, d=128, block=64, new=1, hist=8100, window=2000,
             sinks=4, idle=3, ragged=7),
        # ragged prompts behind cached tokens, window of 1000: compute-bound
        dict(name="sinks_prompt", op="sinks", seqs=4, heads=32, heads_kv=8, d=128, block=64, new=4000, hist=500, window=1000,
             sinks=4, idle=0, ragged=11),
        # two samples of one short conversation: latency
        dict(name="shared_pair", op="shared", seqs=2, heads=32, heads_kv=8, d=128, block=16, new=1, prefix=1040, hist=60,
             idle=0, ragged=0),
        # a decode step of 64 ragged answers behind one long document, three idle slots
        dict(name="shared_batch", op="shared", seqs=64, heads=32, heads_kv=8, d=128, block=64, new=1, prefix=16000, hist=500,
             idle=3, ragged=7),
        # a few drafted tokens per sequence behind a common instruction, 40 full heads
        dict(name="shared_draft", op="shared", seqs=16, heads=40, heads_kv=40, d=128, block=16, new=5, prefix=2000, hist=300,
             idle=0, ragged=9),
        # ragged questions enter behind a document that is in the cache: compute-bound
        dict(name="shared_prompt", op="shared", seqs=8, heads=32, heads_kv=8, d=128, block=64, new=600, prefix=8000, hist=0,
             idle=0, ragged=5),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "rope", "rope_bwd", "sinks_token", "sinks_draft", "sinks_prompt", "shared_token", "shared_draft",
                     "shared_prompt"])
    block = rng.choice([16, 32, 64, 128])
    if op == "plan":
        c = dict(op=op, what=rng.choice(["extend", "extend", "truncate"]), seqs=_log(rng, 1, 4000), block=block)
        c["new"] = _log(rng, 1, max(1, min(4001, 900 * 701 // c["seqs"])))
        c["hist"] = rng.choice([0, _log(rng, 1, max(1, min(8000, 2500 * 900 // c["seqs"])))])
        c["pinned"] = rng.choice([0, 0, rng.randint(0, c["hist"] // block)])
        c["pad"] = rng.choice([0, 0, _log(rng, 1, 200)])
        c["ragged"] = rng.randrange(1, 1 << 20)
        return c
    heads_kv, group = rng.choice([(8, 4), (32, 1), (40, 1), (8, 8), (1, 16), (4, 7)])
    d = rng.choice([64, 128, 128])
    c = dict(op=op.split("_")[0], heads=heads_kv * group, heads_kv=heads_kv, d=d)
    if op.startswith("rope"):
        c["bwd"] = op == "rope_bwd"
        most = 16384 * 80 * 128 // (c["heads"] + heads_kv) // d // (3 if c["bwd"] else 1)
        c["T"] = _log(rng, 1, min(32768, most))
        c["rot"] = rng.choice([d, d, d // 2])
        c["interleaved"], c["norm"] = rng.random() < 0.3, rng.random() < 0.6
        c["base"] = rng.choice([10000.0, 500000.0, 1000000.0])
        c["far"], c["run"] = rng.choice([0, _log(rng, 1, 1000000)]), _log(rng, 1, 8192)
        return c
    c["block"], c["idle"], c["ragged"] = block, 0, rng.randrange(1, 1 << 20)
    kind = op.split("_")[1]
    c["new"] = 1 if kind == "token" else _log(rng, 2, 32) if kind == "draft" else _log(rng, 33, 4000 if c["op"] == "sinks" else 1200)
    if c["op"] == "sinks":
        c["hist"] = rng.choice([0, _log(rng, 1, 4000)]) if kind == "prompt" else _log(rng, 1, 131001)
        c["window"], c["sinks"] = _log(rng, 1, 4096), rng.choice([0, 1, 4, 4, 16, _log(rng, 1, 300)])
        length = c["new"] + c["hist"]
        # the plain form's scores and keys at most the listed cases'
        room = min(4 * 4000 * 4500 * 32 // (c["heads"] * c["new"] * length), 64 * 8100 * 8 // (heads_kv * length))
        if room < 1:
            c["hist"] //= 64
            room = 1
    else:
        c["prefix"] = block * max(1, _log(rng, 16, 32000 if kind == "token" else 8000) // block)
        c["hist"] = rng.choice([0, _log(rng, 1, 2000)])
        length = c["prefix"] + c["hist"] + c["new"]
        # at most the listed prompt's scores
        room = min(8 * 600 * 8600 * 32 // (c["heads"] * c["new"] * length),
                   64 * 16500 * 8 // (heads_kv * (c["hist"] + c["new"] + c["prefix"] // 64)))
    if room < 1:
        c["new"] = max(1, c["new"] // 16)
        room = 1
    c["seqs"] = _log(rng, 1, max(1, min(64, room)))
    if c["seqs"] > 2 and c["new"] == 1:
        c["idle"] = rng.choice([0, 1])
    return c


def lengths(case):
    """Per sequence (tokens in the cache with the new ones, new tokens); the last `idle` slots hold no sequence,
    so their one row is at no position."""
    rng = random.Random(case["ragged"])
    new, hist, prefix = case["new"], case["hist"], case.get("prefix", 0)
    out = []
    for b in range(case["seqs"]):
        if b >= case["seqs"] - case["idle"]:
            out.append((0, 1))
        elif b == 0 or not case["ragged"]:
            out.append((prefix + hist + new, new))
        else:
            n = rng.randint((new + 1) // 2, new)
            out.append((prefix + rng.randint(0, hist) + n, n))
    return out


def requests(case):
    """Of `plan`, per sequence (tokens before, tokens added or, where negative, rows of padding; tokens kept by a
    truncation).  A pinned prefix is in the cache before."""
    rng = random.Random(case["ragged"])
    least = case["pinned"] * case["block"]
    out = []
    for b in range(case["seqs"]):
        before = rng.randint(least, max(least, case["hist"]))
        new = rng.randint((case["new"] + 1) // 2, case["new"])
        if case["what"] == "truncate":
            before += new
        kept = rng.choice([least, before, before - rng.randint(0, min(new, before - least))])
        out.append((before, -1 if rng.random() < 0.05 else new, kept))
    return out


def _blocks(tokens, block):
    return -(-tokens // block)


def taken(case):
    """Blocks that each sequence of `plan` takes or gives back."""
    P, pin = case["block"], case["pinned"]
    if case["what"] == "extend":
        return [max(0, _blocks(before + new, P) - max(_blocks(before, P), pin)) if new > 0 else 0
                for before, new, _ in requests(case)]
    return [max(0, _blocks(before, P) - max(_blocks(kept, P), pin)) for before, _, kept in requests(case)]


def pairs(case):
    """Pairs (query, key) that the mask leaves, over all sequences, and the keys that have to be read."""
    total, keys = 0, case.get("prefix", 0)
    for length, n in lengths(case):
        if length == 0:
            continue
        first, last = length - n, length - 1
        if case["op"] == "shared":
            total += (first + 1 + last + 1) * n // 2
            keys += length - case["prefix"]
            continue
        w, s = case["window"], case["sinks"]
        for p in (first, last) if n == 1 else range(first, last + 1):
            total += min(p + 1, w + min(s, max(0, p + 1 - w)))
        if n == 1:
            total -= min(last + 1, w + min(s, max(0, last + 1 - w)))
        keys += length - max(0, max(0, first - w + 1) - s)
    return total, keys


def work(case):
    if case["op"] == "plan":
        n, rows = case["seqs"], case["pad"] + sum(abs(new) for _, new, _ in requests(case))
        if case["what"] == "truncate":
            return {"bytes": 12 * n + 8 * sum(taken(case)), "flops": 4 * n}
        # lengths and requests in; lengths (the batch's and the sequences') and row starts, positions and slots out;
        # free blocks into the tables
        return {"bytes": 20 * n + 12 * rows + 8 * sum(taken(case)), "flops": 4 * rows}
    if case["op"] == "rope":
        n = case["T"] * (case["heads"] + case["heads_kv"]) * case["d"]
        # the gradient reads x only where it has a norm
        per = (6 if case["norm"] else 4) if case["bwd"] else 4
        return {"bytes": per * n + 4 * case["T"], "flops": (14 if case["bwd"] else 8) * n}
    d, hkv, P = case["d"], case["heads_kv"], case["block"]
    rows = sum(n for _, n in lengths(case))
    seen, keys = pairs(case)
    return {"bytes": 2 * keys * hkv * d + 8 * _blocks(keys, P) * hkv + 4 * rows * case["heads"] * d,
            "flops": 4 * seen * case["heads"] * d}


# ---------------------------------------------------------------------------- inputs
def _int(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _prepare_plan(st, case, g):
    P, pin = case["block"], case["pinned"]
    reqs = requests(case)
    before = [_blocks(b, P) for b, _, _ in reqs]
    need = taken(case)
    width = max(max(_blocks(b + max(0, new), P) for b, new, _ in reqs), 1) + 2
    held = pin + sum(max(0, n - pin) for n in before)
    free = sum(need) + 7 if case["what"] == "extend" else 7
    # a running server's tables: ids in no order, and what earlier sequences left behind their ends
    pool = held + free
    order = torch.randperm(pool, generator=g, device="cuda").int()
    host, at = torch.zeros(case["seqs"], width, dtype=torch.int32), pin
    ids = order.cpu()
    for b, n in enumerate(before):
        host[b, :pin] = ids[:pin]
        own_blocks = max(0, n - pin)
        host[b, pin:pin + own_blocks] = ids[at:at + own_blocks]
        at += own_blocks
    st["table"] = host.cuda()
    st["free"] = torch.cat([order[held:], torch.zeros(pool - free, dtype=torch.int32, device="cuda")])
    st["free_count"] = _int([free])
    # which sequence asks for how much differs from seed to seed
    st["lens"], st["add"], st["keep"] = (_int([r[i] for r in reqs]) for i in range(3))
    turn = torch.randperm(case["seqs"], generator=g, device="cuda")
    for name in ("lens", "add", "keep", "table"):
        st[name] = st[name][turn].contiguous()
    st["rows"] = case["pad"] + sum(abs(new) for _, new, _ in reqs)


def _prepare_rope(st, case, g):
    T, d = case["T"], case["d"]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    heads = case["heads"] + 2 * case["heads_kv"]
    # queries and keys are parts of one projection's output; a few channels are much larger than the others
    channel = torch.where(torch.rand(heads, d, generator=g, device="cuda") < 0.02, 8.0, 1.0)
    qkv = (normal(T, heads, d) * channel).bfloat16()
    st["Q"], st["K"] = qkv[:, :case["heads"]], qkv[:, case["heads"]:case["heads"] + case["heads_kv"]]
    st["gamma"] = [(1.0 + 0.2 * normal(d)).bfloat16() if case["norm"] else None for _ in range(2)]
    if case["bwd"]:
        st["dY"] = [normal(T, h, d).bfloat16() for h in (case["heads"], case["heads_kv"])]
    runs = -(-T // case["run"])
    start = torch.randint(0, case["far"] + 1, (runs,), generator=g, device="cuda")
    t = torch.arange(T, device="cuda")
    st["pos"] = (start[t // case["run"]] + t % case["run"]).int()
    st["freq"] = [case["base"] ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]
    if own:
        st["rope"] = _rope(st)


def _prepare_attn(st, case, g):
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    hkv, d, P = case["heads_kv"], case["d"], case["block"]
    ls = lengths(case)
    first = case.get("prefix", 0) // P
    blocks = [max(0, _blocks(length, P) - first) for length, _ in ls]
    width = max(1, first + max(blocks))
    pool = first + sum(blocks) + 3
    order = torch.randperm(pool, generator=g, device="cuda").int()
    at, tables = first, torch.zeros(case["seqs"], width, dtype=torch.int32, device="cuda")
    for b, n in enumerate(blocks):
        if ls[b][0]:
            tables[b, :first] = order[:first]
        tables[b, first:first + n] = order[at:at + n]
        at += n
    st["table"] = tables
    st["prefix_table"] = order[:first].clone()
    st["rows"] = sum(n for _, n in ls)
    st["max_new"] = max(n for _, n in ls)
    st["max_len"] = max(length for length, _ in ls)
    start = [0]
    for _, n in ls:
        start.append(start[-1] + n)
    st["lens"], st["start"] = _int([length for length, _ in ls]), _int(start)
    # a block's largest magnitude is its scale times 127; keys have a few large channels
    for name in ("k", "v"):
        codes = normal(pool, hkv, P, d)
        if name == "k":
            codes *= torch.where(torch.rand(hkv, 1, d, generator=g, device="cuda") < 0.03, 4.0, 1.0)
        amax = codes.abs().amax((2, 3))
        st[name + "_codes"] = (codes * (127.0 / amax)[:, :, None, None]).round().to(torch.int8)
        st[name + "_scale"] = amax / 127.0
    # queries as the first part of a projection's output that also holds keys and values
    qkv = normal(st["rows"], case["heads"] + 2 * hkv, d).bfloat16()
    st["Q"] = qkv[:, :case["heads"]]
    st["scale"] = 1.5 / math.sqrt(d)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case)
    {"plan": _prepare_plan, "rope": _prepare_rope}.get(case["op"], _prepare_attn)(st, case, g)
    return st


# ---------------------------------------------------------------------------- the plain forms
def _plan(st):
    P, pin = st["block"], st["pinned"]
    lens, table, free, count = st["lens"].long(), st["table"], st["free"], st["free_count"].long()
    up = lambda n: torch.div(n + P - 1, P, rounding_mode="floor")  # noqa: E731
    column = torch.arange(table.shape[1], device="cuda")
    if st["what"] == "truncate":
        kept = torch.minimum(lens, st["keep"].long().clamp(min=0))
        lo = up(kept).clamp(min=pin)[:, None]
        back = (column >= lo) & (column < up(lens)[:, None])
        total = back.sum()
        order = torch.cumsum(back.flatten().long(), 0) - 1
        at = torch.where(back.flatten(), count + total - 1 - order, free.shape[0])
        longer = torch.cat([free, free.new_zeros(1)]).scatter_(0, at, table.flatten())
        free.copy_(longer[:-1])
        return [kept.int(), (count + total).int(), free]
    add = st["add"].long()
    new = add.clamp(min=0)
    end = torch.cumsum(add.abs(), 0)
    start = torch.cat([end.new_zeros(1), end])
    lo = up(lens).clamp(min=pin)
    need = torch.where(new > 0, (up(lens + new) - lo).clamp(min=0), 0)
    base = torch.cumsum(need, 0) - need
    taken_ = (column >= lo[:, None]) & (column < (lo + need)[:, None])
    at = (count - 1 - base)[:, None] - (column - lo[:, None])
    table.copy_(torch.where(taken_, free[torch.where(taken_, at, 0)], table))
    row = torch.arange(st["rows"], device="cuda")
    b = torch.searchsorted(end, row, right=True)
    inside = b < add.shape[0]
    b = torch.where(inside, b, 0)
    inside = inside & (add[b] > 0)
    pos = torch.where(inside, lens[b] + row - start[b], -1)
    slot = torch.where(inside, table[b, pos.clamp(min=0) // P].long() * P + pos % P, -1)
    return [(lens + new).int(), torch.where(add > 0, lens + new, torch.where(add < 0, 0, lens)).int(), start.int(),
            (count - need.sum()).int(), table, pos.int(), slot]


def _turn(x, cos, sin, rot, interleaved):
    """Rotates the pairs of the first `rot` elements of each head x [T, heads, d]."""
    cos, sin = cos[:, None], sin[:, None]
    rest = x[..., rot:]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, rest], -1)


def _rope_plain(st):
    angle = st["pos"].double()[:, None] * _int(st["freq"], torch.float64)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out, dgamma = [], []
    for i, name in enumerate("QK"):
        x, gamma = st[name].float(), st["gamma"][i]
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) if gamma is not None else None
        if not st["bwd"]:
            n = x * r * gamma.float() if gamma is not None else x
            out.append(_turn(n, cos, sin, st["rot"], st["interleaved"]).bfloat16())
            continue
        g = _turn(st["dY"][i].float(), cos, -sin, st["rot"], st["interleaved"])
        if gamma is not None:
            dgamma.append((g * x * r).sum((0, 1)))
            g = g * gamma.float()
            g = r * (g - x * (r * r * (g * x).mean(-1, keepdim=True)))
        out.append(g.bfloat16())
    return out + dgamma


def _places(lens, start, rows):
    """Sequence, row within it and position in it of each of `rows` rows (the newest of each sequence)."""
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(start.long(), r, right=True) - 1
    i = r - start.long()[b]
    return b, i, lens.long()[b] - (start[1:] - start[:-1]).long()[b] + i


def _values(st, name, table):
    """Keys or values behind a block table [..., blocks] as [..., heads, blocks * P, d]."""
    v = st[name + "_codes"][table].float() * st[name + "_scale"][table][..., None, None]
    v = v.transpose(-4, -3)
    return v.reshape(*v.shape[:-3], -1, st["d"])


def _attn(st):
    hkv, d, P, n = st["heads_kv"], st["d"], st["block"], st["max_new"]
    B, group, prefix = st["seqs"], st["heads"] // st["heads_kv"], st.get("prefix", 0)
    b, i, pos = _places(st["lens"], st["start"], st["rows"])
    q = torch.zeros(B, n, hkv, group, d, device="cuda")
    q[b, i] = st["Q"].float().reshape(-1, hkv, group, d)
    q = q.permute(0, 2, 1, 3, 4) * st["scale"]                     # [B, hkv, n, group, d]
    at = torch.full((B, n), -1, device="cuda")
    at[b, i] = pos
    # the sequences' own keys, from position `prefix` on
    table = st["table"].long()[:, prefix // P:]
    own_keys = table.shape[1] * P
    j = prefix + torch.arange(own_keys, device="cuda")
    sees = j <= at[:, :, None]
    if st["op"] == "sinks":
        sees = sees & ((j > at[:, :, None] - st["window"]) | (j < st["sinks"]))
    s = torch.matmul(q.reshape(B, hkv, n * group, d), _values(st, "k", table).transpose(-1, -2))
    s = torch.where(sees[:, None, :, None], s.view(B, hkv, n, group, own_keys), -INF)
    m = s.amax(-1, keepdim=True) if own_keys else torch.full((B, hkv, n, group, 1), -INF, device="cuda")
    if prefix:
        # keys that all share: one product for every row of the batch
        rows = q.transpose(0, 1).reshape(hkv, B * n * group, d)
        sp = torch.matmul(rows, _values(st, "k", st["prefix_table"].long()).transpose(-1, -2))
        sp = sp.view(hkv, B, n, group, prefix).transpose(0, 1)
        sp = torch.where((torch.arange(prefix, device="cuda") <= at[:, :, None])[:, None, :, None], sp, -INF)
        m = torch.maximum(m, sp.amax(-1, keepdim=True))
    base = torch.where(m > -INF, m, torch.zeros_like(m))
    p = torch.exp(s - base)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, hkv, n * group, own_keys), _values(st, "v", table)).view(B, hkv, n, group, d)
    if prefix:
        p = torch.exp(sp - base)
        total = total + p.sum(-1, keepdim=True)
        p = p.transpose(0, 1).reshape(hkv, B * n * group, prefix)
        o = o + torch.matmul(p, _values(st, "v", st["prefix_table"].long())).view(hkv, B, n, group, d).transpose(0, 1)
    o = o / torch.where(total > 0, total, 1.0)
    return [o.permute(0, 2, 1, 3, 4)[b, i].reshape(-1, st["heads"], d).bfloat16()]


# ---------------------------------------------------------------------------- the framework's operators
def _rope(st):
    from paper_2406_06385_gb300 import lrqat as LQ
    return LQ.QKRope.of(st["heads"], st["heads_kv"], st["d"], LQ.rope_turns(st["freq"]).cuda(), st["interleaved"], EPS)


def _own(st):
    from paper_2406_06385_gb300 import lrqat as LQ
    new = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if st["op"] == "plan":
        n = st["seqs"]
        blocks = LQ.KVBlocks.of(st["table"], st["free"], st["block"], st["pinned"])
        lens, left = new(n, dtype=torch.int32), new(1, dtype=torch.int32)
        ws = new(LQ.kv_blocks_workspace_bytes(blocks), dtype=torch.uint8)
        if st["what"] == "truncate":
            LQ.kv_truncate(blocks, st["lens"], st["keep"], st["free_count"], lens, left, ws)
            return [lens, left, st["free"]]
        seen, start = new(n, dtype=torch.int32), new(n + 1, dtype=torch.int32)
        pos, slot = new(st["rows"], dtype=torch.int32), new(st["rows"], dtype=torch.int64)
        LQ.kv_extend(blocks, st["lens"], st["add"], st["free_count"], lens, left, seen, start, pos, slot, ws)
        return [lens, seen, start, left, st["table"], pos, slot]
    if st["op"] == "rope":
        rope = st["rope"] if "rope" in st else _rope(st)
        T, d = st["T"], st["d"]
        Q, K = new(T, st["heads"], d), new(T, st["heads_kv"], d)
        if not st["bwd"]:
            LQ.qk_rope_fwd(rope, st["pos"], st["Q"], st["K"], *st["gamma"], Q, K)
            return [Q, K]
        norm = st["norm"]
        dgamma = [new(d, dtype=torch.float32) if norm else None for _ in range(2)]
        ws = new(LQ.qk_rope_bwd_workspace_bytes(rope, T), dtype=torch.uint8) if norm else None
        x = (st["Q"], st["K"]) if norm else (None, None)
        LQ.qk_rope_bwd(rope, st["pos"], *st["dY"], *x, *st["gamma"], Q, K, *dgamma, False, ws)
        return [Q, K] + (dgamma if norm else [])
    cache = LQ.KVCache.of(st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"])
    batch = LQ.KVBatch.of(st["lens"], st["start"], st["table"], st["rows"], st["max_new"], st["max_len"])
    O = new(st["rows"], st["heads"], st["d"])
    if st["op"] == "sinks":
        ws = new(LQ.kv_attn_sinks_workspace_bytes(cache, batch, st["heads"], st["window"], st["sinks"]), dtype=torch.uint8)
        LQ.kv_attn_sinks(cache, batch, st["Q"], st["scale"], st["window"], st["sinks"], O, ws)
    else:
        ws = new(LQ.kv_attn_shared_workspace_bytes(cache, batch, st["heads"], st["prefix"]), dtype=torch.uint8)
        LQ.kv_attn_shared(cache, batch, st["prefix_table"], st["prefix"], st["Q"], st["scale"], O, ws)
    return [O]


def run(state):
    if own:
        return _own(state)
    return {"plan": _plan, "rope": _rope_plain}.get(state["op"], _attn)(state)


# ---------------------------------------------------------------------------- 64 bits
def _exact_plan(st):
    P, pin = st["block"], st["pinned"]
    lens, add, keep = (st[name].tolist() for name in ("lens", "add", "keep"))
    table, free, count = st["table"].tolist(), st["free"].tolist(), int(st["free_count"])
    if st["what"] == "truncate":
        back, kept = [], []
        for row, length, k in zip(table, lens, keep):
            kept.append(min(length, max(0, k)))
            back += row[max(-(-kept[-1] // P), pin):-(-length // P)]
        free[count:count + len(back)] = back[::-1]
        return [_int(kept), _int([count + len(back)]), _int(free)]
    seen, start, pos, slot, after = [], [0], [], [], []
    for row, length, a in zip(table, lens, add):
        start.append(start[-1] + abs(a))
        after.append(length + max(0, a))
        seen.append(after[-1] if a >= 0 else 0)
        for p in range(length, length + a):
            if p % P == 0 and p // P >= pin:
                count -= 1
                row[p // P] = free[count]
            pos.append(p)
            slot.append(row[p // P] * P + p % P)
        pos += [-1] * -a
        slot += [-1] * -a
    pos += [-1] * (st["rows"] - len(pos))
    slot += [-1] * (st["rows"] - len(slot))
    return [_int(after), _int(seen), _int(start), _int([count]), _int(table), _int(pos), _int(slot, torch.int64)]


def _exact_rope(st):
    D = torch.float64
    rot, half = st["rot"], st["rot"] // 2
    # the rotation as a product of complex numbers
    unit = torch.polar(torch.ones(1, dtype=D, device="cuda"), st["pos"].to(D)[:, None] * _int(st["freq"], D))[:, None]
    first = torch.arange(0, rot, 2, device="cuda") if st["interleaved"] else torch.arange(half, device="cuda")
    second = first + (1 if st["interleaved"] else half)
    out, dgamma = [], []
    for i, name in enumerate("QK"):
        x, gamma = st[name].to(D), st["gamma"][i]
        y = st["dY"][i].to(D) if st["bwd"] else x
        if gamma is not None:
            rms = torch.sqrt(torch.linalg.vecdot(x, x)[..., None] / st["d"] + EPS)
            x = x / rms
            if not st["bwd"]:
                y = x * gamma.to(D)
        z = torch.complex(y[..., first], y[..., second]) * (unit.conj() if st["bwd"] else unit)
        y = y.clone()
        y[..., first], y[..., second] = z.real, z.imag
        if st["bwd"] and gamma is not None:
            dgamma.append(torch.einsum("thd,thd->d", y, x))
            y = y * gamma.to(D)
            y = (y - x * torch.linalg.vecdot(x, y)[..., None] / st["d"]) / rms
        out.append(y)
    return out + dgamma


def _exact_attn(st, case):
    D = torch.float64
    P, hkv, d = case["block"], case["heads_kv"], case["d"]
    start, group = st["start"].tolist(), case["heads"] // hkv
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
            key = torch.arange(length, device="cuda")
            far = pos[:, None] - key
            hidden = far < 0
            if case["op"] == "sinks":
                hidden |= (far >= case["window"]) & (key >= case["sinks"])
            s = torch.einsum("rhgd,hkd->hgrk", q[rows], k) * st["scale"]
            out[rows] = torch.einsum("hgrk,hkd->rhgd", torch.softmax(s.masked_fill(hidden, -INF), -1), v)
    return [out.view(st["rows"], -1, d)]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "plan":
        return _exact_plan(st)
    if case["op"] == "rope":
        return _exact_rope(st)
    return _exact_attn(st, case)
