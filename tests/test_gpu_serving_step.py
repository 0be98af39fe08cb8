"""The operators of a serving step run together, as the attention example runs them: blocks from the device's own list, norm and
rotation of each head, cache, attention (through a window with sinks, or behind a shared prefix), blocks given back.

Tolerance of the block: that of test_gpu_attention_example.py, whose roundings are the same; the rotated queries and keys
are rounded to bf16 once more (2^-8), which is within what the projection's 1e-2 leaves.  Of the operators alone: those of
their own tests, each step on the device's inputs."""
import numpy as np
import pytest

import oracle as O
from oracle import serving_oracle as SO
from paper_2406_06385_gb300 import lrqat as LQ

from gpu_util import bits_to_f32, empty, to_dev, torch
from test_gpu_attention_example import RefProjection, _bf16, _np, _quant, example  # noqa: F401
from test_gpu_kv_step_attn import _bound

pytestmark = pytest.mark.gpu


def _ints(v):
    return to_dev(np.asarray(v, np.int32))


class Ref:
    """The block in float64 on the oracle's cache; blocks and lengths are the oracle's own."""

    def __init__(self, blk, running, freq, prefix):
        self.blk, self.freq, self.prefix, self.eps = blk, freq, prefix, blk.rope.eps
        c, P = running.cache, running.blocks.block
        self.caches = [SO.Cache(c.n_blocks, blk.kv_heads, P, blk.d) for _ in range(2)]
        self.blocks = SO.Blocks(running.table.cpu().numpy(), running.blocks.tensors[1].cpu().numpy(), int(running.free),
                                [0] * running.length.numel(), P, running.blocks.pinned)
        self.qkv, self.out = RefProjection(blk.qkv), RefProjection(blk.out)

    def step(self, x, res, seqs, tables, pos, eps, window=0, sinks=0):
        """seqs: (length, rows) in the order of the rows; length 0: padding."""
        blk, h = self.blk, _np(x) + _np(res)
        y = self.qkv.forward(_quant(SO.rmsnorm(h, _np(blk.gamma_in), eps))).reshape(len(pos), -1, blk.d)
        at, live = blk.heads, np.asarray(pos) >= 0
        turn = lambda v, g: np.where(live[:, None, None], _bf16(SO.head_norm_rope(  # noqa: E731
            v, None if g is None else _np(g), np.maximum(pos, 0), self.freq, self.eps)), v)
        q, k, v = turn(y[:, :at], blk.gamma_q), turn(y[:, at:at + blk.kv_heads], blk.gamma_k), y[:, at + blk.kv_heads:]
        a, r0 = np.zeros(q.shape), 0
        for (length, n), table in zip(seqs, tables):
            rows = slice(r0, r0 + n)
            r0 += n
            if length == 0:
                continue
            for c, new in zip(self.caches, (k, v)):
                c.write(new[rows], length, table)
            a[rows] = SO.attention(q[rows], *[c.values(length, table) for c in self.caches], length, 1 / np.sqrt(blk.d), window,
                                   sinks)[0]
        h2 = self.out.forward(_quant(_bf16(a).reshape(len(pos), -1))) + _bf16(h)
        return h2, _quant(SO.rmsnorm(h2, _np(blk.gamma_out), eps))


@pytest.mark.parametrize("shared", [False, True])
def test_block_of_running_sequences(example, shared):  # noqa: F811
    t = torch()
    t.manual_seed(6)
    hidden, heads, kv_heads, d, P, prefix = 256, 4, 2, 64, 16, 48 if shared else 0
    freq = [10000.0 ** (-2 * i / d) for i in range(d // 2)]
    vec = lambda n: (1 + 0.2 * t.randn(n, device="cuda")).bfloat16()  # noqa: E731
    rope = LQ.QKRope.of(heads, kv_heads, d, LQ.rope_turns(freq).cuda())
    blk = example.AttentionBlock(example.random_projection((heads + 2 * kv_heads) * d, hidden),
                                 example.random_projection(hidden, heads * d), vec(hidden), vec(hidden), heads, kv_heads, d, rope,
                                 vec(d), vec(d))
    run = example.RunningSequences(4, 160, 60, kv_heads, d, P, prefix // P)
    ref = Ref(blk, run, freq, prefix)
    rows = lambda n: [t.randn(n, hidden, device="cuda").bfloat16() for _ in range(2)]  # noqa: E731

    def same(got, want):
        LQ.get_device_status()
        assert O.rel_fro(_np(got[0]), want[0]) <= 2e-2 and O.rel_fro(_np(got[1]), want[1]) <= 2e-2

    if shared:
        x, pos = rows(prefix), np.arange(prefix)
        alone = LQ.KVBatch.of(_ints([prefix]), _ints([0, prefix]), run.prefix_table[None], prefix, prefix, prefix)
        same(blk.step(*x, run.cache, alone, pos=_ints(pos)),
             ref.step(*x, [(prefix, prefix)], [run.prefix_table.cpu().numpy()], pos, example.EPS))
        run.length.fill_(prefix)
        ref.blocks.len = [prefix] * 4
    window, sinks = (0, 0) if shared else (20, 4)
    kw = dict(prefix_table=run.prefix_table) if shared else dict(window=window, sinks=sinks)
    for new, drop in (([37, 1, 70, 5], [0, 0, 0, 0]), ([1, 1, 1, -1], [0, 0, 0, 0]), ([4, 3, 4, 4], [2, 0, 4, 1]),
                      ([1, 9, 1, 2], [0, 200, 0, 0]), ([2, 20, 1, 1], [0, 0, 0, 0])):
        n = sum(abs(m) for m in new)
        batch, pos = run.append(_ints(new), n, max(new))
        lens, start, at, _, refused = ref.blocks.extend(new, n)
        assert not refused and pos.tolist() == at and run.start.tolist() == start
        x = rows(n)
        same(blk.step(*x, run.cache, batch, pos=pos, **kw),
             ref.step(*x, [(m, abs(a)) for m, a in zip(lens, new)], ref.blocks.table, at, example.EPS, window, sinks))
        keep = [max(m - k, prefix) for m, k in zip(ref.blocks.len, drop)]
        run.shorten(_ints(keep))
        ref.blocks.truncate(keep)
        assert run.length.tolist() == ref.blocks.len and int(run.free) == ref.blocks.free
        assert np.array_equal(run.table.cpu().numpy(), ref.blocks.table)


@pytest.mark.parametrize("shared", [False, True])
def test_captured_decode_steps(shared):
    """One captured step, replayed with other inputs and other requests; two more graphs of it, on another stream, share
    its workspaces."""
    t = torch()
    rng = np.random.default_rng(8)
    n_seqs, hq, hk, d, P, rows, prefix = 6, 32, 8, 128, 16, 32, 8000 if shared else 0
    freq = [500000.0 ** (-2 * i / d) for i in range(d // 2)]
    rope = LQ.QKRope.of(hq, hk, d, LQ.rope_turns(freq).cuda())
    pool, width, pin = 120 + prefix // P, 24 + prefix // P, prefix // P
    codes = [t.randint(-127, 128, (pool, hk, P, d), dtype=t.int8, device="cuda") for _ in range(2)]
    scale = [t.rand(pool, hk, device="cuda") * 0.02 + 0.001 for _ in range(2)]
    cache = LQ.KVCache.of(*codes, *scale)
    ids = rng.permutation(pool).astype(np.int32)
    table = np.full((n_seqs, width), 10 ** 6, np.int32)
    table[:, :pin] = ids[pool - pin:]
    table_d, prefix_table, length = _ints(table), _ints(ids[pool - pin:]), _ints([prefix] * n_seqs)
    free, add, seen, start = _ints([pool - pin]), _ints([0] * n_seqs), _ints([0] * n_seqs), _ints([0] * (n_seqs + 1))
    pos = _ints([0] * rows)
    blocks = LQ.KVBlocks.of(table_d, _ints(ids), P, pin)
    batch = LQ.KVBatch.of(seen, start, table_d, rows, 16, width * P)
    qkv = t.zeros((rows, hq + 2 * hk, d), dtype=t.bfloat16, device="cuda")
    q, k, v = qkv.split([hq, hk, hk], 1)
    turned = t.zeros((rows, hq + hk, d), dtype=t.bfloat16, device="cuda")
    qr, kr = turned.split([hq, hk], 1)
    out = t.zeros((rows, hq, d), dtype=t.bfloat16, device="cuda")
    need = LQ.kv_attn_shared_workspace_bytes(cache, batch, hq, prefix) if shared else LQ.kv_attn_sinks_workspace_bytes(
        cache, batch, hq, 40, 4)
    ws, room = empty((max(need, 16),), t.uint8), empty((LQ.kv_blocks_workspace_bytes(blocks),), t.uint8)
    s = 1.4 / np.sqrt(d)

    def step():
        LQ.kv_extend(blocks, length, add, free, length, free, seen, start, pos, None, room)
        LQ.qk_rope_fwd(rope, pos, q, k, None, None, qr, kr)
        LQ.kv_write(cache, batch, kr, v)
        if shared:
            LQ.kv_attn_shared(cache, batch, prefix_table, prefix, qr, s, out, ws)
        else:
            LQ.kv_attn_sinks(cache, batch, qr, s, 40, 4, out, ws)

    step()                                                    # nothing is asked for
    graphs, side = [], t.cuda.Stream()
    for i in range(3):
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            step()
        graphs.append(g)
    for turn in range(7):
        a = rng.integers(1, 6, n_seqs)
        a[rng.integers(n_seqs)] = (-1, 0)[turn % 2]
        add.copy_(_ints(a))
        qkv.copy_(t.randn(qkv.shape, device="cuda").bfloat16())
        out.fill_(float("nan"))
        if turn % 3:
            side.wait_stream(t.cuda.current_stream())
            with t.cuda.stream(side):
                graphs[turn % 3].replay()
            t.cuda.current_stream().wait_stream(side)
        else:
            graphs[0].replay()
        LQ.get_device_status()
        p, L, r0 = pos.cpu().numpy(), seen.tolist(), start.tolist()
        assert [b - c for b, c in zip(r0[1:], r0)] == np.abs(a).tolist()
        live = p >= 0
        x = _np(qkv[:, :hq])
        ref = SO.rotate(x[live], p[live], freq)
        assert (np.abs(_np(qr)[live] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * np.abs(x[live]).max()).all()
        vals = [(c.float() * m[..., None, None]).double().cpu().numpy() for c, m in zip(codes, scale)]
        tab, got, qn = table_d.cpu().numpy(), _np(out), _np(qr)
        for b in range(n_seqs):
            sl = slice(r0[b], r0[b + 1])
            kk, vv = (np.concatenate([m[i].transpose(1, 0, 2) for i in tab[b, :-(-L[b] // P)]] or [np.zeros((0, hk, d))])[:L[b]]
                      for m in vals)
            want, mass, n = SO.attention(qn[sl], kk, vv, L[b], s, 0 if shared else 40, 0 if shared else 4)
            assert (np.abs(got[sl] - want) <= _bound(want, mass, n, np.abs(vv).max(initial=0.0))).all()
        assert np.isnan(got[r0[-1]:]).all()                   # rows behind the last sequence stay as they were
