"""GPU parity of the head norm and rotation and of its gradient, against numpy in float64.

Tolerances.  Forward, with (a, b) the normed pair: the output's rounding to bf16, 2^-8 |y|; the norm's fp32 arithmetic
(a sum of squares in chains of at most 20 additions, a root, a division, two products: below 2^-19 of |n|) and the
angle's (its fraction rounded to 24 bits, 2^-22 rad, sine and cosine within two units: below 2^-20), together below
2^-18 (|a| + |b|).  Backward, with s = |dy_a| + |dy_b| of a pair: 2^-8 |dx| and 2^-18 of the same sums of magnitudes,
r (s |gamma| + |x| r^2 mean(s |gamma x|)); dgamma: 2^-18 of the sum of |terms|, and 2^-24 of it for each of N terms."""
import numpy as np
import pytest

from oracle import serving_oracle as SO
from paper_2406_06385_gb300 import lrqat as LQ
from paper_2406_06385_gb300 import workloads as WL

from gpu_util import bits_to_f32, empty, to_dev, torch

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _bf16(rng, *shape, spread=1.0):
    x = rng.standard_normal(shape) * 10.0 ** rng.uniform(-spread, spread, shape[:-1] + (1,))
    bits = WL.bf16_bits(x.astype(np.float32))
    return bits, WL.bf16_to_f32(bits).astype(np.float64)


def _freq(rot, base=10000.0):
    return [base ** (-2.0 * i / rot) for i in range(rot // 2)]


def _gammas(rng, d, norm):
    g = [_bf16(rng, d, spread=0.0) if n else (None, None) for n in norm]
    return [None if b is None else to_dev(b) for b, _ in g], [v for _, v in g]


def _pair_sum(x, rot, neighbours):
    """|a| + |b| of the pair that each element belongs to; the element's own magnitude where it passes."""
    s = np.abs(x)
    a, b = (s[..., 0:rot:2], s[..., 1:rot:2]) if neighbours else (s[..., :rot // 2], s[..., rot // 2:rot])
    both = a + b
    out = s.copy()
    if neighbours:
        out[..., 0:rot:2] = out[..., 1:rot:2] = both
    else:
        out[..., :rot // 2] = out[..., rot // 2:rot] = both
    return out


def _normed(x, gamma):
    return x if gamma is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * gamma


SHAPES = [
    # T, query heads, key heads, d, rot, neighbours, (query norm, key norm)
    (1, 32, 8, 128, 128, False, (True, True)),
    (1, 1, 1, 64, 64, False, (False, False)),
    (3, 5, 1, 128, 64, False, (True, False)),
    (7, 40, 40, 128, 128, True, (False, False)),
    (33, 28, 4, 64, 32, True, (True, True)),
    (20, 3, 2, 16, 16, False, (True, True)),
    (21, 2, 3, 32, 32, True, (False, True)),
    (19, 7, 1, 80, 48, False, (True, True)),
    (19, 3, 1, 96, 96, True, (True, True)),
    (40, 2, 2, 256, 256, False, (True, True)),
    (11, 4, 1, 240, 64, False, (True, True)),
    (50, 4, 2, 128, 0, False, (True, True)),
    (17, 9, 0, 128, 128, False, (True, False)),
    (17, 0, 9, 64, 64, False, (False, True)),
    (3001, 2, 1, 64, 64, False, (True, True)),
]


def _setup(T, hq, hk, d, rot, neighbours, norm, seed):
    rng = np.random.default_rng(seed)
    freq = _freq(rot)
    rope = LQ.QKRope.of(hq, hk, d, LQ.rope_turns(freq).cuda() if rot else None, neighbours, EPS)
    pos = rng.integers(0, 2 ** rng.integers(1, 32, T), dtype=np.int64).clip(0, 2 ** 31 - 1).astype(np.int32)
    g_dev, g = _gammas(rng, d, norm)
    return rng, freq, rope, pos, g_dev, g


@pytest.mark.parametrize("T,hq,hk,d,rot,neighbours,norm", SHAPES)
def test_forward(T, hq, hk, d, rot, neighbours, norm):
    rng, freq, rope, pos, g_dev, g = _setup(T, hq, hk, d, rot, neighbours, norm, T + d)
    t = torch()
    x = [_bf16(rng, T, h, d) for h in (hq, hk)]
    src = [to_dev(b) if h else None for (b, _), h in zip(x, (hq, hk))]
    out = [t.full((T, h, d), 0x7FC0, dtype=t.int16, device="cuda") if h else None for h in (hq, hk)]
    LQ.qk_rope_fwd(rope, to_dev(pos), *src, *g_dev, *out)
    LQ.get_device_status()
    for i, o in enumerate(out):
        if o is None:
            continue
        ref = SO.head_norm_rope(x[i][1], g[i], pos, freq, EPS, neighbours)
        bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * _pair_sum(_normed(x[i][1], g[i]), rot, neighbours)
        assert (np.abs(bits_to_f32(o) - ref) <= bound).all()
    # in place, as views of one projection's output, gives the same bits
    both = t.zeros((T, hq + hk + 3, d), dtype=t.int16, device="cuda")
    views = [both[:, :hq] if hq else None, both[:, hq + 2:hq + 2 + hk] if hk else None]
    for v, s in zip(views, src):
        if v is not None:
            v.copy_(s)
    rest = both[:, hq:hq + 2].clone()
    LQ.qk_rope_fwd(rope, to_dev(pos), *views, *g_dev, *views)
    for v, o in zip(views, out):
        assert v is None or t.equal(v, o)
    assert t.equal(both[:, hq:hq + 2], rest) and (both[:, hq + hk + 2:] == 0).all()


@pytest.mark.parametrize("T,hq,hk,d,rot,neighbours,norm", SHAPES)
def test_backward(T, hq, hk, d, rot, neighbours, norm):
    rng, freq, rope, pos, g_dev, g = _setup(T, hq, hk, d, rot, neighbours, norm, T + d + 1)
    t = torch()
    heads = (hq, hk)
    x, dy = ([_bf16(rng, T, h, d) for h in heads] for _ in range(2))
    dev = lambda v, i: to_dev(v[i][0]) if heads[i] else None  # noqa: E731
    want = [n and h > 0 for n, h in zip(norm, heads)]
    dgamma = [t.full((d,), 3.0, device="cuda") if w else None for w in want]
    out = [t.full((T, h, d), 0x7FC0, dtype=t.int16, device="cuda") if h else None for h in heads]
    ws = empty((LQ.qk_rope_bwd_workspace_bytes(rope, T),), t.uint8)
    ws.fill_(0xFF)
    args = [dev(dy, 0), dev(dy, 1), dev(x, 0) if want[0] else None, dev(x, 1) if want[1] else None, *g_dev]
    LQ.qk_rope_bwd(rope, to_dev(pos), *args, *out, *dgamma, False, ws)
    LQ.get_device_status()
    for i in range(2):
        if not heads[i]:
            continue
        ref, dg = SO.head_norm_rope_bwd(dy[i][1], x[i][1], g[i], pos, freq, EPS, neighbours)
        s, xx = _pair_sum(dy[i][1], rot, neighbours), np.abs(x[i][1])
        if g[i] is None:
            bound = 2.0 ** -18 * s
        else:
            r = 1.0 / np.sqrt((xx * xx).mean(-1, keepdims=True) + EPS)
            bound = 2.0 ** -18 * r * (s * np.abs(g[i]) + xx * r * r * (s * np.abs(g[i]) * xx).mean(-1, keepdims=True))
            terms = (s * xx * r).sum((0, 1))
            assert (np.abs(dgamma[i].cpu().numpy() - dg) <= (2.0 ** -18 + T * heads[i] * 2.0 ** -24) * terms).all()
        assert (np.abs(bits_to_f32(out[i]) - ref) <= 2.0 ** -8 * np.abs(ref) + bound).all()
    # again, in place over the upstream gradients: the same bits; accumulating adds the same sums
    dgamma2 = [None if v is None else v.clone() for v in dgamma]
    LQ.qk_rope_bwd(rope, to_dev(pos), *args, args[0], args[1], *dgamma2, True, ws)
    for i in range(2):
        assert out[i] is None or t.equal(args[i], out[i])
        assert dgamma[i] is None or t.equal(dgamma2[i], dgamma[i] + dgamma[i])


@pytest.mark.parametrize("T,hq,hk,d", [(20011, 8, 1, 128), (60001, 1, 1, 64)])
def test_dgamma_of_many_terms(T, hq, hk, d):
    """Sums of up to 160088 terms.  However they are ordered, one of n terms in a chain of additions per lane, with lanes,
    warps and blocks joined by trees and short chains behind it, is off by at most 2^-24 of the terms' magnitudes for each
    addition that a term goes through: here the lane's own (two blocks of 8 warps an SM, a warp's lanes 512 elements at a
    time), at most 4 among a warp's heads, 8 among warps, a 32nd of the blocks, 5 in the tree, one to accumulate.  A term
    itself is off by 2^-18, as above."""
    rng, freq, rope, pos, g_dev, g = _setup(T, hq, hk, d, d, False, (True, True), T)
    t = torch()
    heads = (hq, hk)
    x, dy = ([_bf16(rng, T, h, d) for h in heads] for _ in range(2))
    dgamma = [t.zeros(d, device="cuda") for _ in range(2)]
    ws = empty((LQ.qk_rope_bwd_workspace_bytes(rope, T),), t.uint8)
    out = [t.empty((T, h, d), dtype=t.int16, device="cuda") for h in heads]
    LQ.qk_rope_bwd(rope, to_dev(pos), *[to_dev(v[0]) for v in dy + x], *g_dev, *out, *dgamma, False, ws)
    LQ.get_device_status()
    blocks = 2 * t.cuda.get_device_properties(0).multi_processor_count
    for i, h in enumerate(heads):
        _, dg = SO.head_norm_rope_bwd(dy[i][1], x[i][1], g[i], pos, freq, EPS)
        s, xx = _pair_sum(dy[i][1], d, False), np.abs(x[i][1])
        terms = (s * xx / np.sqrt((xx * xx).mean(-1, keepdims=True) + EPS)).sum((0, 1))
        lane = -(-T // (8 * blocks)) * -(-h * d // 512)
        depth = lane + 4 + 8 + -(-blocks // 32) + 5 + 1
        assert (np.abs(dgamma[i].cpu().numpy() - dg) <= (2.0 ** -18 + depth * 2.0 ** -24) * terms).all()


def test_rows_without_a_position():
    """pos None is row t at position t; rows at negative positions stay as they were in the forward and have a zero gradient
    (their inputs may be anything) that adds nothing to dgamma."""
    t = torch()
    rng = np.random.default_rng(5)
    T, h, d = 37, 3, 64
    freq = _freq(d)
    rope = LQ.QKRope.of(h, h, d, LQ.rope_turns(freq).cuda(), False, 0.0)
    src = [to_dev(_bf16(rng, T, h, d)[0]) for _ in range(4)]
    gamma = to_dev(_bf16(rng, d, spread=0.0)[0])
    new = lambda: [t.full((T, h, d), 77, dtype=t.int16, device="cuda") for _ in range(2)]  # noqa: E731
    a, b = new(), new()
    LQ.qk_rope_fwd(rope, None, *src[:2], gamma, None, *a)
    LQ.qk_rope_fwd(rope, to_dev(np.arange(T, dtype=np.int32)), *src[:2], gamma, None, *b)
    assert all(t.equal(x, y) for x, y in zip(a, b))
    pos = np.arange(T, dtype=np.int32)
    pad = np.array([0, 4, 5, 36])
    pos[pad] = [-1, -2 ** 31, -5, -1]
    live = np.setdiff1d(np.arange(T), pad)
    for s in src:                                          # NaN, and heads of zeros (eps is 0)
        s[pad[0]] = 0x7FC0
        s[pad[1]] = 0
    c = new()
    LQ.qk_rope_fwd(rope, to_dev(pos), *src[:2], gamma, None, *c)
    assert all(t.equal(x[live], y[live]) and (x[pad] == 77).all() for x, y in zip(c, a))
    ws = empty((LQ.qk_rope_bwd_workspace_bytes(rope, T),), t.uint8)
    dgs = []
    for rows, p in ((slice(None), pos), (live, pos[live])):
        dx, dg = new(), t.zeros(d, device="cuda")
        dx = [v[rows].contiguous() for v in dx]
        part = [s[rows].contiguous() for s in src]
        LQ.qk_rope_bwd(rope, to_dev(p), *part[2:], part[0], None, gamma, None, *dx, dg, None, False, ws)
        dgs.append((dx, dg))
    (dx, dg), (dx_live, dg_live) = dgs
    assert all((v[pad] == 0).all() and t.equal(v[live], w) for v, w in zip(dx, dx_live))
    assert t.allclose(dg, dg_live, rtol=0, atol=2.0 ** -14 * float(dg_live.abs().max()) + 1e-3) and t.isfinite(dg).all()


def test_far_positions_keep_their_angle():
    """Neighbouring positions close to 2^31 differ by the angle of one step; negative and fast frequencies."""
    t = torch()
    freq = [1.0, -0.7, 3.0e-4, 1234.5, 6.25, 1e-9, 2.0 ** 20, 0.0]
    rope = LQ.QKRope.of(1, 0, 16, LQ.rope_turns(freq).cuda(), False, 0.0)
    pos = np.array([0, 1, 2 ** 24 + 1, 2 ** 31 - 2, 2 ** 31 - 1], np.int32)
    x = np.zeros((5, 1, 16), np.float32)
    x[..., :8] = 1.0                                       # the outputs are cosines and sines
    out = t.zeros((5, 1, 16), dtype=t.int16, device="cuda")
    LQ.qk_rope_fwd(rope, to_dev(pos), to_dev(WL.bf16_bits(x)), None, None, None, out, None)
    from fractions import Fraction
    pi = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803")
    got = bits_to_f32(out)
    for i, p in enumerate(pos):
        for j, f in enumerate(freq):
            w = float(Fraction(f) * int(p) % (2 * pi))
            ref = np.array([np.cos(w), np.sin(w)])
            assert (np.abs(got[i, 0, [j, 8 + j]] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18).all()


def test_infinite_and_nan_heads_stay_in_their_heads():
    t = torch()
    rng = np.random.default_rng(6)
    rope = LQ.QKRope.of(8, 2, 128, LQ.rope_turns(_freq(128)).cuda())
    bits, _ = _bf16(rng, 9, 8, 128)
    k, _ = _bf16(rng, 9, 2, 128)
    gamma = to_dev(_bf16(rng, 128, spread=0.0)[0])
    out = [t.zeros((9, h, 128), dtype=t.int16, device="cuda") for h in (8, 2)]
    ref = [v.clone() for v in out]
    LQ.qk_rope_fwd(rope, None, to_dev(bits), to_dev(k), gamma, gamma, *ref)
    bad = bits.copy()
    bad[3, 2, 7], bad[8, 7, 127] = 0x7FC0, 0x7F80
    LQ.qk_rope_fwd(rope, None, to_dev(bad), to_dev(k), gamma, gamma, *out)
    hit = np.zeros((9, 8), bool)
    hit[3, 2] = hit[8, 7] = True
    got = bits_to_f32(out[0])
    assert np.isnan(got[3, 2]).all() and np.isnan(got[8, 7, [63, 127]]).all()
    assert np.array_equal(got[~hit], bits_to_f32(ref[0])[~hit]) and t.equal(out[1], ref[1])


def test_other_streams_graphs_and_repeated_backwards():
    """A captured forward and backward replayed on other positions and inputs, on a side stream; the sums of dgamma do not
    depend on the run."""
    t = torch()
    rng = np.random.default_rng(7)
    T, hq, hk, d = 500, 8, 2, 128
    freq = _freq(d, 500000.0)
    rope = LQ.QKRope.of(hq, hk, d, LQ.rope_turns(freq).cuda(), False, EPS)
    gamma = [to_dev(_bf16(rng, d, spread=0.0)[0]) for _ in range(2)]
    pos = t.zeros(T, dtype=t.int32, device="cuda")
    x, dy, y, dx = ([t.zeros((T, h, d), dtype=t.int16, device="cuda") for h in (hq, hk)] for _ in range(4))
    dg = [t.zeros(d, device="cuda") for _ in range(2)]
    ws = empty((LQ.qk_rope_bwd_workspace_bytes(rope, T),), t.uint8)

    def both():
        LQ.qk_rope_fwd(rope, pos, *x, *gamma, *y)
        LQ.qk_rope_bwd(rope, pos, *dy, *x, *gamma, *dx, *dg, False, ws)

    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        both()
    side.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        both()
    for turn in range(3):
        pos.copy_(to_dev(rng.integers(0, 1 << 20, T).astype(np.int32)))
        for v in x + dy:
            v.copy_(to_dev(_bf16(rng, *v.shape)[0]))
        graph.replay()
        t.cuda.synchronize()
        kept = [v.clone() for v in y + dx + dg]
        for v in y + dx + dg:
            v.zero_()
        both()
        assert all(t.equal(a, b) for a, b in zip(kept, y + dx + dg))


def test_many_tokens_pass_32_bit_offsets():
    """Rows whose elements lie more than 2^31 elements and 2^32 bytes into their arrays, as parts of wide rows."""
    t = torch()
    T, wide = 70000, 32768                                 # 4.6 GB of bf16
    base = t.zeros((T, wide), dtype=t.int16, device="cuda")
    q, k = base[:, 64:192].unflatten(1, (2, 64)), base[:, 256:320].unflatten(1, (1, 64))
    rng = np.random.default_rng(8)
    rows = np.array([0, 1, 65535, 65536, 69999])
    bits = _bf16(rng, 5, 3, 64)[0]
    q[rows] = to_dev(bits[:, :2])
    k[rows] = to_dev(bits[:, 2:])
    rope = LQ.QKRope.of(2, 1, 64, LQ.rope_turns(_freq(64)).cuda())
    LQ.qk_rope_fwd(rope, None, q, k, None, None, q, k)
    few = [to_dev(bits[:, :2]), to_dev(bits[:, 2:])]
    LQ.qk_rope_fwd(rope, to_dev(rows.astype(np.int32)), *few, None, None, *few)
    assert t.equal(q[rows], few[0]) and t.equal(k[rows], few[1])
    assert int(((base & 0x7FFF) != 0).sum()) <= 5 * 3 * 64                 # zeros elsewhere, of either sign
