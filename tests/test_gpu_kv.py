"""GPU parity of the 8-bit cache's writes and reads (codes and scales bit for bit) and of attention over it,
against numpy.

Tolerance of attention, per element of an output o = sum_j p_j v_j: half a bf16 ulp of o (2^-9 |o|); half an ulp
of the 11-bit probabilities, fp32 scores with their exponential and fp32 sums (together below 2^-11 sum_j p_j |v_j|);
and 2^-25 of the largest contribution for each of the n keys (probabilities below the half-precision range),
times codes up to 127: n 2^-18 max_j(p_j s_v,j) <= n 2^-18 max(o's scale)."""
import numpy as np
import pytest

from oracle import serving_oracle as SO
from paper_2406_06385_gb300 import lrqat as LQ
from paper_2406_06385_gb300 import workloads as WL

from gpu_util import bits_to_f32, empty, to_dev, torch

pytestmark = pytest.mark.gpu


class Paged:
    """Sequences (length, new rows) in a pool of blocks handed out in random order; device and oracle caches."""

    def __init__(self, seqs, heads, d, block, seed=0, spare=2, first_block=0):
        t = torch()
        self.rng = np.random.default_rng(seed)
        self.seqs, self.heads, self.d, self.block = seqs, heads, d, block
        need = [-(-length // block) for length, _ in seqs]
        pool = first_block + sum(need) + spare
        ids = first_block + self.rng.permutation(sum(need) + spare)
        self.table = np.full((len(seqs), max(1, max(need))), -7, np.int32)       # unused entries are never followed
        self.blocks, at = [], 0
        for b, n in enumerate(need):
            self.blocks.append([int(i) for i in ids[at:at + n]])
            self.table[b, :n] = ids[at:at + n]
            at += n
        shape = (pool, heads, block, d)
        self.codes = [t.full(shape, 85, dtype=t.int8, device="cuda") for _ in range(2)]      # never cleared memory
        self.scale = [t.full(shape[:2], float("nan"), device="cuda") for _ in range(2)]
        self.cache = LQ.KVCache.of(self.codes[0], self.codes[1], self.scale[0], self.scale[1])

    def batch(self, seqs=None, slack=0):
        seqs = self.seqs if seqs is None else seqs
        start = np.concatenate([[0], np.cumsum([n for _, n in seqs])]).astype(np.int32)
        max_len = min(max(length for length, _ in seqs) + slack, self.table.shape[1] * self.block)
        return LQ.KVBatch.of(to_dev(np.array([length for length, _ in seqs], np.int32)), to_dev(start),
                             to_dev(self.table), int(start[-1]), max(n for _, n in seqs) + slack, max_len)

    def random_rows(self, heads, seqs=None, scale=1.0):
        n = sum(n for _, n in (self.seqs if seqs is None else seqs))
        x = self.rng.standard_normal((n, heads, self.d)) * scale
        x *= 10.0 ** self.rng.uniform(-1, 1, (n, 1, 1))
        bits = WL.bf16_bits(x.astype(np.float32))
        return bits, WL.bf16_to_f32(bits)


def _seq_rows(seqs):
    at = 0
    for b, (length, n) in enumerate(seqs):
        yield b, length, n, slice(at, at + n)
        at += n


@pytest.mark.parametrize("heads,d,block,steps", [
    (2, 128, 16, [[(1, 1), (17, 17), (40, 40)], [(2, 1), (18, 1), (41, 1)], [(35, 33), (31, 13), (41, 0)]]),
    (1, 64, 16, [[(33, 33)], [(34, 1)], [(48, 14)], [(49, 1)]]),
    (3, 128, 64, [[(63, 63), (64, 64), (0, 1)], [(64, 1), (65, 1), (0, 1)], [(200, 136), (66, 1), (5, 9)]]),
    (5, 64, 128, [[(1, 1), (300, 300)], [(129, 128), (301, 1)]]),
    (2, 128, 32, [[(10, 10)], [(12, 2)], [(13, 1)], [(95, 82)]])])
def test_writes_and_reads_bit_exact(heads, d, block, steps):
    """Several calls fill the sequences: single tokens, chunks that start and end inside blocks, idle slots and padding
    rows; larger tokens make the scales of started blocks grow."""
    final = [(max(s[b][0] for s in steps), 0) for b in range(len(steps[0]))]
    p = Paged(final, heads, d, block, seed=d + block)
    oracle = [SO.Cache(p.cache.n_blocks, heads, block, d) for _ in range(2)]
    for c in oracle:
        c.codes[:] = 85
    for turn, seqs in enumerate(steps):
        rows = [p.random_rows(heads, seqs, scale=1.0 + turn) for _ in range(2)]
        batch = p.batch(seqs, slack=turn)
        for _ in range(2):                                      # writing again changes nothing
            LQ.kv_write(p.cache, batch, to_dev(rows[0][0]), to_dev(rows[1][0]))
        LQ.get_device_status()
        for kv in range(2):
            for b, length, n, at in _seq_rows(seqs):
                take = min(n, length)
                x = rows[kv][1][at][n - take:]
                if take:
                    oracle[kv].write(x, length, p.blocks[b])
            assert np.array_equal(p.scale[kv].cpu().numpy(), oracle[kv].scale, equal_nan=True)
            assert np.array_equal(p.codes[kv].cpu().numpy(), oracle[kv].codes)
    # whole sequences back
    seqs = [(length, length) for length, _ in final]
    n = sum(length for length, _ in seqs)
    K, V = (torch().zeros((n, heads, d), dtype=torch().int16, device="cuda") for _ in range(2))
    LQ.kv_read(p.cache, p.batch(seqs), K, V)
    LQ.get_device_status()
    for kv, got in enumerate((K, V)):
        for b, length, _, at in _seq_rows(seqs):
            ref = oracle[kv].values(length, p.blocks[b])
            assert np.array_equal(bits_to_f32(got)[at], WL.bf16_to_f32(WL.bf16_bits(ref.astype(np.float32))))


def test_write_from_parts_of_a_projection_and_read_into_parts():
    t = torch()
    p = Paged([(37, 37), (5, 5)], 4, 128, 16, seed=3)
    both, _ = p.random_rows(12)
    proj = to_dev(both)
    LQ.kv_write(p.cache, p.batch(), proj[:, 4:8], proj[:, 8:])
    codes, scale = [c.clone() for c in p.codes], [s.clone() for s in p.scale]
    LQ.kv_write(p.cache, p.batch(), proj[:, 4:8].contiguous(), proj[:, 8:].contiguous())
    assert all(t.equal(a, b) for a, b in zip(codes, p.codes))
    assert all(t.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(scale, p.scale))
    out, dense = t.zeros_like(proj), [t.zeros((42, 4, 128), dtype=t.int16, device="cuda") for _ in range(2)]
    LQ.kv_read(p.cache, p.batch(), out[:, 8:], out[:, :4])
    LQ.kv_read(p.cache, p.batch(), *dense)
    assert t.equal(out[:, 8:], dense[0]) and t.equal(out[:, :4], dense[1]) and (out[:, 4:8] == 0).all()


def test_zeros_tiny_and_not_finite_values():
    t = torch()
    p = Paged([(64, 64)], 2, 64, 16, seed=4)
    x = np.zeros((64, 2, 64), np.float32)
    x[16:32, 0] = 1e-38                                   # its scale is subnormal
    x[16, 0, 1] = 3e-38
    x[20, 1, 3] = np.inf
    x[40, 0, 0] = 5.0
    bits = WL.bf16_bits(x)
    bits[50, 1, 7] = 0x7FC0                               # NaN
    LQ.kv_write(p.cache, p.batch(), to_dev(bits), to_dev(bits))
    LQ.get_device_status()
    K, V = (t.zeros((64, 2, 64), dtype=t.int16, device="cuda") for _ in range(2))
    LQ.kv_read(p.cache, p.batch(), K, V)
    k = bits_to_f32(K)
    s = p.scale[0].cpu().numpy()[p.blocks[0]]
    assert s[0].tolist() == [1, 1] and (k[:16] == 0).all()
    assert (np.abs(k[16:32, 0] - x[16:32, 0]) <= 0.51 * s[1, 0] + 2.0 ** -8 * x[16:32, 0]).all()
    assert np.isnan(s[1, 1]) and np.isnan(k[16:32, 1]).all()
    assert np.isnan(s[3, 1]) and np.isnan(k[48:, 1]).all() and (k[48:, 0] == 0).all()
    assert k[40, 0, 0] == WL.bf16_to_f32(WL.bf16_bits(np.float32([127 * s[2, 0]])))[0]


# ---------------------------------------------------------------------------- attention
def _fill(p, kv_scale=None):
    """Random codes and scales for the sequences' blocks; other blocks keep NaN scales.  Returns the values."""
    t = torch()
    used = np.array(sorted(i for bl in p.blocks for i in bl), np.int64)
    host = []
    for kv in range(2):
        codes = np.clip(np.rint(p.rng.standard_normal((len(used), p.heads, p.block, p.d)) * 45), -128, 127).astype(np.int8)
        scale = (10.0 ** p.rng.uniform(-2.2, -1.5, (len(used), p.heads))).astype(np.float32)
        if kv_scale is not None:
            scale = kv_scale(kv, used, scale)
        p.codes[kv][t.from_numpy(used).cuda()] = t.from_numpy(codes).cuda()
        p.scale[kv][t.from_numpy(used).cuda()] = t.from_numpy(scale).cuda()
        host.append((codes, scale))
    slot = {int(b): i for i, b in enumerate(used)}
    vals = []
    for b, (length, _) in enumerate(p.seqs):
        ids = [slot[i] for i in p.blocks[b]]
        vals.append([(c[ids].astype(np.float64) * s[ids].astype(np.float64)[:, :, None, None]).transpose(0, 2, 1, 3)
                     .reshape(-1, p.heads, p.d)[:length] for c, s in host])
    return vals


def _attn(p, batch, Q, scale, window, n_heads, out=None, stream=None):
    t = torch()
    O = t.full(Q.shape, 0x7FC0, dtype=t.int16, device="cuda") if out is None else out
    ws = empty((LQ.kv_attn_workspace_bytes(p.cache, batch, n_heads, window),), t.uint8)
    ws.fill_(0xFF)
    LQ.kv_attn(p.cache, batch, Q, scale, window, O, ws, stream=stream)
    return O


def _check(p, vals, O, q, scale, window):
    got = bits_to_f32(O).astype(np.float64)
    for b, length, n, at in _seq_rows(p.seqs):
        ref, mass, seen = SO.attention(q[at], *vals[b], length, scale, window)
        top = np.abs(vals[b][1]).max(initial=0.0)
        bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -11 * mass + (seen[:, None, None] * 2.0 ** -25) * top
        bad = ~(np.abs(got[at] - ref) <= bound)
        assert not bad.any(), (b, np.argwhere(bad)[:5], got[at][bad][:5], ref[bad][:5])


CASES = [
    # sequences (length, new), kv heads, group, d, block, window
    ([(1, 1)], 1, 1, 128, 16, 0),
    ([(1, 1), (15, 1), (16, 1), (17, 1), (64, 1), (65, 1), (129, 1)], 2, 4, 128, 16, 0),
    ([(1000, 1), (0, 1), (333, 1), (2049, 1)], 8, 4, 128, 64, 0),
    ([(700, 1), (90, 1)], 5, 1, 64, 32, 0),
    ([(300, 1), (31, 1)], 1, 16, 64, 128, 0),
    ([(300, 2), (31, 1)], 2, 7, 128, 16, 0),
    ([(130, 3), (64, 1)], 1, 71, 128, 16, 0),
    ([(40, 40), (5, 5), (77, 30)], 2, 4, 128, 16, 0),
    ([(200, 130), (257, 257)], 1, 1, 128, 128, 0),
    ([(150, 129), (128, 128)], 2, 2, 64, 64, 0),
    ([(3, 9), (20, 21), (0, 4), (50, 2)], 2, 4, 128, 16, 0),         # padding rows before the first position
    ([(100, 5), (33, 33), (2000, 1)], 2, 4, 128, 32, 1),
    ([(100, 5), (33, 33), (2000, 2)], 2, 1, 128, 32, 17),
    ([(500, 200), (333, 300)], 1, 2, 64, 16, 64),
    ([(900, 64), (1500, 3)], 2, 8, 128, 64, 511),
    ([(20000, 1)], 1, 8, 128, 128, 0),
    ([(9000, 4)], 2, 1, 128, 16, 0),
]


@pytest.mark.parametrize("seqs,heads,group,d,block,window", CASES)
def test_attention(seqs, heads, group, d, block, window):
    p = Paged(seqs, heads, d, block, seed=len(seqs) + block)
    vals = _fill(p)
    bits, q = p.random_rows(heads * group)
    scale = 1.3 / np.sqrt(d)
    O = _attn(p, p.batch(), to_dev(bits), scale, window, heads * group)
    LQ.get_device_status()
    _check(p, vals, O, q, scale, window)
    t = torch()
    assert t.equal(O, _attn(p, p.batch(), to_dev(bits), scale, window, heads * group))


@pytest.mark.parametrize("new", [1, 40])
def test_windows_as_long_as_the_sequences_hide_nothing(new):
    t = torch()
    p = Paged([(300, new), (77, new)], 2, 128, 16, seed=16)
    vals = _fill(p)
    bits, q = p.random_rows(8)
    O = _attn(p, p.batch(), to_dev(bits), 0.1, 0, 8)
    _check(p, vals, O, q, 0.1, 0)
    for window in (300, 301, 2 ** 31 - 1):
        assert t.equal(O, _attn(p, p.batch(), to_dev(bits), 0.1, window, 8))


def test_many_short_sequences():
    """Hundreds of sequences of all small lengths, a third of them idle slots."""
    rng = np.random.default_rng(17)
    seqs = [(0, 1) if i % 3 == 2 else (int(rng.integers(1, 70)), 1) for i in range(400)]
    p = Paged(seqs, 4, 64, 16, seed=17)
    vals = _fill(p)
    bits, q = p.random_rows(8)
    O = _attn(p, p.batch(), to_dev(bits), 0.2, 0, 8)
    LQ.get_device_status()
    _check(p, vals, O, q, 0.2, 0)


@pytest.mark.parametrize("longest", [2048, 2049, 2000])
@pytest.mark.parametrize("new,window", [(1, 0), (2, 0), (1, 1024)])
def test_sequences_that_end_where_pieces_do(longest, new, window):
    """Lengths at, before and behind the ends of the pieces that the keys are cut into (multiples of 128 and
    256 here), next to idle slots and to a longest sequence with and without a short last piece."""
    lens = [n for m in (128, 256, 512, 1024, 1920) for n in (m - 1, m, m + 1)] + [new, longest]
    p = Paged([(n, new) for n in lens] + [(0, new)], 1, 128, 16, seed=longest + new)
    vals = _fill(p)
    bits, q = p.random_rows(4)
    O = _attn(p, p.batch(), to_dev(bits), 0.1, window, 4)
    LQ.get_device_status()
    _check(p, vals, O, q, 0.1, window)


@pytest.mark.parametrize("seqs", [[(700, 1), (40, 1)], [(300, 150)]])
def test_attention_with_scales_far_apart(seqs):
    """Blocks whose scales lie many orders of magnitude apart: values as large as 1e20 behind negligible weights, tiny
    values behind the whole weight."""
    p = Paged(seqs, 2, 128, 16, seed=8)

    def far(kv, used, scale):
        if kv == 1:
            scale = (10.0 ** p.rng.uniform(-20, 20, scale.shape)).astype(np.float32)
        return scale

    vals = _fill(p, far)
    bits, q = p.random_rows(4)
    O = _attn(p, p.batch(), to_dev(bits), 0.5, 0, 4)
    LQ.get_device_status()
    got = bits_to_f32(O).astype(np.float64)
    for b, length, n, at in _seq_rows(p.seqs):
        ref, mass, seen = SO.attention(q[at], *vals[b], length, 0.5)
        # the largest contribution p_j |v_j| is at most the mass; scores of magnitude z carry z 2^-22 into p
        z = 0.5 * np.abs(np.einsum("nhd,lhd->nhl", q[at].astype(np.float64), np.repeat(vals[b][0], 2, 1))).max()
        bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + (z + 100) * 2.0 ** -21 + seen[:, None, None] * 2.0 ** -18) * mass.max(2, keepdims=True)
        assert (np.abs(got[at] - ref) <= bound).all()


def test_attention_queries_of_any_magnitude():
    """Rows of q from 1e-30 to 1e30 with a softmax scale to match: q is scaled by a power of two per row."""
    p = Paged([(200, 9)], 2, 128, 32, seed=9)
    vals = _fill(p)
    _, q = p.random_rows(4)
    for mag in (1e-30, 1e30):
        bits = WL.bf16_bits((q * mag).astype(np.float32))
        qq = WL.bf16_to_f32(bits)
        scale = float(np.float32(0.1 / mag))
        O = _attn(p, p.batch(), to_dev(bits), scale, 0, 4)
        LQ.get_device_status()
        _check(p, vals, O, qq, scale, 0)


@pytest.mark.parametrize("new", [1, 6, 100])
def test_hidden_blocks_do_not_leak(new):
    """Blocks outside a row's window hold NaN scales, and the rest of the last block garbage codes: neither reaches the
    result.  A NaN scale inside the window makes the row NaN."""
    window, length = 48, 400
    p = Paged([(length, new)], 2, 128, 16, seed=10)
    vals = _fill(p)
    first = max(0, length - new - window + 1)
    for kv in range(2):
        for i in range(first // 16):
            p.scale[kv][p.blocks[0][i]] = float("nan")
    bits, q = p.random_rows(4)
    O = _attn(p, p.batch(), to_dev(bits), 0.1, window, 4)
    LQ.get_device_status()
    _check(p, vals, O, q, 0.1, window)
    p.scale[1][p.blocks[0][-1]] = float("nan")
    got = bits_to_f32(_attn(p, p.batch(), to_dev(bits), 0.1, window, 4))
    assert np.isnan(got[-1]).all()
    if new == 100:                # early rows do not see the last block
        sees = np.arange(length - new, length) >= length - 16
        assert np.isnan(got[sees]).all() and not np.isnan(got[~sees]).any()


def test_infinite_and_nan_queries_stay_in_their_rows():
    p = Paged([(100, 8)], 1, 128, 16, seed=11)
    vals = _fill(p)
    bits, q = p.random_rows(2)
    bad = bits.copy()
    bad[3, 1, 5], bad[6, 0, 9] = 0x7FC0, 0x7F80
    got = bits_to_f32(_attn(p, p.batch(), to_dev(bad), 0.1, 0, 2))
    ref = bits_to_f32(_attn(p, p.batch(), to_dev(bits), 0.1, 0, 2))
    hit = np.zeros((8, 2), bool)
    hit[3, 1] = hit[6, 0] = True
    assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], ref[~hit])


@pytest.mark.parametrize("seqs,heads,group,block,window", [
    ([(1030, 1)], 8, 4, 16, 0), ([(40000, 1), (33000, 1)], 8, 4, 32, 0), ([(9000, 4), (5000, 4)], 8, 4, 64, 0),
    ([(3000, 5)] * 3, 16, 1, 16, 2048), ([(6000, 1)] * 6 + [(200, 1)] * 6, 8, 1, 128, 0), ([(4000, 300)], 4, 4, 64, 0)])
def test_results_do_not_depend_on_where_the_cache_lies(seqs, heads, group, block, window):
    """The same bits whether the cache comes from memory (a buffer larger than the L2 cache was written before) or
    from L2, and close to float64: no copy is used before it has arrived."""
    t = torch()
    p = Paged(seqs, heads, 128, block, seed=15)
    vals = _fill(p)
    bits, q = p.random_rows(heads * group)
    Q, batch = to_dev(bits), p.batch()
    junk = t.empty(1 << 28, dtype=t.float32, device="cuda")
    out = []
    for i in range(6):
        if i < 4:
            junk.fill_(float(i))
        out.append(_attn(p, batch, Q, 0.1, window, heads * group))
    LQ.get_device_status()
    assert all(t.equal(o, out[0]) for o in out)
    got = bits_to_f32(out[0]).astype(np.float64)
    at = 0
    for b, (length, n) in enumerate(seqs):
        row = slice(at + n - 1, at + n)                     # the newest row of each sequence
        at += n
        ref, mass, seen = SO.attention(q[row], *vals[b], length, 0.1, window)
        bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -11 * mass + (seen[:, None, None] * 2.0 ** -25) * np.abs(vals[b][1]).max()
        assert (np.abs(got[row] - ref) <= bound).all()


def test_strided_rows_other_streams_and_graphs():
    """Q and O as parts of wider rows; the call on a side stream; a captured call replayed for other lengths within the
    captured bounds."""
    t = torch()
    seqs = [(70, 1), (200, 1), (16, 1)]
    p = Paged([(length + 60, 1) for length, _ in seqs], 2, 128, 16, seed=12)
    vals = _fill(p)
    p.seqs = seqs
    bits, q = p.random_rows(8)
    wide = t.zeros((3, 16, 128), dtype=t.int16, device="cuda")
    wide[:, 4:12] = to_dev(bits)
    out = t.zeros((3, 20, 128), dtype=t.int16, device="cuda")
    batch = p.batch(slack=60)
    ref = _attn(p, batch, to_dev(bits), 0.1, 0, 8)
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        _attn(p, batch, wide[:, 4:12], 0.1, 0, 8, out=out[:, 8:16])
    side.synchronize()
    assert t.equal(out[:, 8:16], ref) and (out[:, :8] == 0).all() and (out[:, 16:] == 0).all()
    lens = batch.tensors[0]
    Q, O = to_dev(bits), t.zeros((3, 8, 128), dtype=t.int16, device="cuda")
    ws = empty((LQ.kv_attn_workspace_bytes(p.cache, batch, 8, 0),), t.uint8)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        LQ.kv_attn(p.cache, batch, Q, 0.1, 0, O, ws)
    for add in (0, 37, 60, -16):
        lens.copy_(t.tensor([length + add for length, _ in seqs], dtype=t.int32))
        graph.replay()
        t.cuda.synchronize()
        p.seqs = [(length + add, 1) for length, _ in seqs]
        cut = [[v[:length + add] for v in vals[b]] for b, (length, _) in enumerate(seqs)]
        _check(p, cut, O, q, 0.1, 0)


def test_blocks_past_two_gigabytes():
    """Cache blocks whose byte offsets need more than 32 bits."""
    p = Paged([(300, 1), (130, 130)], 8, 128, 128, seed=13, first_block=17000)       # 17000 * 128 KiB = 2.2 GB
    seqs = p.seqs
    rows = [p.random_rows(8, [(300, 300), (130, 130)]) for _ in range(2)]
    p.seqs = [(300, 300), (130, 130)]
    LQ.kv_write(p.cache, p.batch(), to_dev(rows[0][0]), to_dev(rows[1][0]))
    vals = []
    oracle = [SO.Cache(p.cache.n_blocks - 17000, 8, 128, 128) for _ in range(2)]
    for b, length, n, at in _seq_rows(p.seqs):
        local = [i - 17000 for i in p.blocks[b]]
        for kv in range(2):
            oracle[kv].write(rows[kv][1][at], length, local)
        vals.append([o.values(length, local) for o in oracle])
    for kv in range(2):
        assert np.array_equal(p.scale[kv][17000:].cpu().numpy(), oracle[kv].scale, equal_nan=True)
    p.seqs = seqs
    bits, q = p.random_rows(16, scale=0.1)
    O = _attn(p, p.batch(), to_dev(bits), 0.05, 0, 16)
    LQ.get_device_status()
    _check(p, vals, O, q, 0.05, 0)


def test_arrays_that_contradict_the_bounds_are_reported():
    """A block id outside the pool, rows beyond the batch, a length beyond the bound: the sequence is skipped, the others
    are served, and the device status says so once."""
    t = torch()
    p = Paged([(40, 1), (50, 1)], 2, 128, 16, seed=14)
    vals = _fill(p)
    bits, q = p.random_rows(4)
    Q = to_dev(bits)

    def expect(batch):
        O = _attn(p, batch, Q, 0.1, 0, 4)
        with pytest.raises(LQ.LrqatError) as e:
            LQ.get_device_status()
        assert e.value.status == -7
        LQ.get_device_status()
        got = bits_to_f32(O).astype(np.float64)
        ref, mass, _ = SO.attention(q[1:2], *vals[1], 50, 0.1)
        assert (np.abs(got[1:2] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mass).all()

    for what, value in (("table", p.cache.n_blocks), ("table", -1), ("lens", 10 ** 6), ("lens", -5)):
        batch = p.batch()
        batch.tensors[{"lens": 0, "table": 2}[what]].view(-1)[0] = value
        expect(batch)
        if what == "table":
            before = [c.clone() for c in p.codes]
            K = to_dev(p.random_rows(2)[0])
            batch.tensors[2][0, -2:] = value              # the block that the new token of sequence 0 goes to
            batch.tensors[2][0, :] = value
            LQ.kv_write(p.cache, batch, K, K)
            with pytest.raises(LQ.LrqatError):
                LQ.get_device_status()
            for kv in range(2):
                moved = (p.codes[kv] != before[kv]).flatten(1).any(1).nonzero().flatten().tolist()
                assert set(moved) <= {p.blocks[1][-1]}
                p.codes[kv].copy_(before[kv])
            _restore(p, vals)
    batch = p.batch()
    batch.rows = 1                                         # the second sequence's row lies outside the call's arrays
    _attn(p, batch, Q, 0.1, 0, 4)
    with pytest.raises(LQ.LrqatError):
        LQ.get_device_status()
    batch = p.batch()
    batch.tensors[1][2] = 5                                # more rows than max_rows
    _attn(p, batch, Q, 0.1, 0, 4)
    with pytest.raises(LQ.LrqatError):
        LQ.get_device_status()


def _restore(p, vals):
    """Scales of the last block of sequence 1 as they were (its codes were copied back)."""
    t = torch()
    for kv in range(2):
        blk = p.blocks[1][-1]
        codes = p.codes[kv][blk].double()                  # [heads, block, d]
        v = t.from_numpy(vals[1][kv][48]).cuda()           # the first token of that block, [heads, d]
        i = codes[:, 0].abs().argmax(1)
        h = t.arange(p.heads, device="cuda")
        p.scale[kv][blk] = (v[h, i] / codes[h, 0, i]).float()


@pytest.mark.parametrize("new", [1, 6, 40])
@pytest.mark.parametrize("length", [100, 5000])
def test_values_that_are_all_zero_give_zero_whatever_the_scores(new, length):
    """Every visible value scale is 0 and every score lies hundreds of powers of two below 0."""
    p = Paged([(length, new)], 2, 128, 16, seed=21)
    _fill(p, lambda kv, used, scale: scale * np.float32(kv == 0))
    p.codes[0].clamp_(min=1)
    bits, q = p.random_rows(4)
    bits |= 0x8000                                         # every element of q is negative
    O = _attn(p, p.batch(), to_dev(bits), 300.0, 0, 4)
    LQ.get_device_status()
    assert (bits_to_f32(O) == 0).all()


@pytest.mark.parametrize("new", [1, 6, 40, 300])
def test_blocks_with_a_value_scale_of_zero_count_in_the_denominator(new):
    """A cache that was quantized elsewhere may hold blocks of zeros with scale 0: their keys take their share of the
    softmax and their values add nothing, whichever kernel the number of rows leads to."""
    p = Paged([(300, new), (47, min(new, 47))], 2, 128, 16, seed=20)

    def zeros(kv, used, scale):
        if kv == 1:
            scale[::2] = 0.0
        return scale

    vals = _fill(p, zeros)
    bits, q = p.random_rows(4)
    O = _attn(p, p.batch(), to_dev(bits), 0.1, 0, 4)
    LQ.get_device_status()
    _check(p, vals, O, q, 0.1, 0)


@pytest.mark.parametrize("seqs", [[(700, 1), (40, 1)], [(300, 150)], [(2000, 70)]])
def test_value_scales_on_both_sides_of_the_first_one(seqs):
    """Blocks 2^63 above and 2^63 below the first one's scale of about 1: the small ones carry as much of the
    denominator as the large ones.  Bound: as for scales far apart."""
    p = Paged(seqs, 2, 128, 16, seed=22)

    def both(kv, used, scale):
        if kv == 0:
            return scale
        slot = {int(i): n for n, i in enumerate(used)}
        for ids in p.blocks:
            for j, i in enumerate(ids):
                scale[slot[i]] = 1.0 if j == 0 else 2.0 ** (63 if j % 2 else -63) * p.rng.uniform(0.6, 0.9)
        return scale

    vals = _fill(p, both)
    bits, q = p.random_rows(4)
    O = _attn(p, p.batch(), to_dev(bits), 0.1, 0, 4)
    LQ.get_device_status()
    got = bits_to_f32(O).astype(np.float64)
    for b, length, n, at in _seq_rows(p.seqs):
        ref, mass, seen = SO.attention(q[at], *vals[b], length, 0.1)
        z = 0.1 * np.abs(np.einsum("nhd,lhd->nhl", q[at].astype(np.float64), np.repeat(vals[b][0], 2, 1))).max()
        bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + (z + 100) * 2.0 ** -21 + seen[:, None, None] * 2.0 ** -18) * mass.max(2, keepdims=True)
        assert (np.abs(got[at] - ref) <= bound).all()


@pytest.mark.parametrize("block,d", [(16, 64), (64, 128)])
def test_tokens_behind_zeros_keep_their_values(block, d):
    """A block whose tokens so far are all zeros takes the scale of the first ones that are not, in a later call as in the
    same one; a block of scale 1 that holds anything else keeps it."""
    t = torch()
    p = Paged([(0, 0), (0, 0)], 2, d, block, seed=23, spare=6)
    p.table = np.array([[1, 2], [4, 3]], np.int32)
    p.blocks = [[1, 2], [4, 3]]
    for c in p.codes:
        c[:] = 85
    oracle = [SO.Cache(p.cache.n_blocks, 2, block, d) for _ in range(2)]
    for c in oracle:
        c.codes[:] = 85
    steps = [([(3, 3), (2, 2)], 0.0, 127.0), ([(4, 1), (3, 1)], 0.0, 1e-2), ([(5, 1), (4, 1)], 1e-3, 1e-2),
             ([(6, 1), (6, 2)], 2e-3, 500.0), ([(7, 1), (7, 1)], 1e-4, 0.0)]
    for seqs, *top in steps:
        n0 = seqs[0][1]
        rows = []
        for _ in range(2):
            x = p.rng.uniform(-1, 1, (n0 + seqs[1][1], 2, d)).astype(np.float32)
            x[0, :, 0] = x[n0, :, 0] = 1.0                 # the largest magnitudes are `top`
            x[:n0] *= top[0]
            x[n0:] *= top[1]
            bits = WL.bf16_bits(x)
            rows.append((bits, WL.bf16_to_f32(bits)))
        for _ in range(2):                                 # writing again changes nothing
            LQ.kv_write(p.cache, p.batch(seqs), to_dev(rows[0][0]), to_dev(rows[1][0]))
        LQ.get_device_status()
        for kv in range(2):
            for b, length, n, at in _seq_rows(seqs):
                oracle[kv].write(rows[kv][1][at], length, p.blocks[b])
            assert np.array_equal(p.scale[kv].cpu().numpy(), oracle[kv].scale, equal_nan=True)
            assert np.array_equal(p.codes[kv].cpu().numpy(), oracle[kv].codes)
    assert (p.scale[0][1] < 1e-4).all() and (p.scale[0][4] > 3).all()


@pytest.mark.parametrize("top", [0.5, 0.0])
def test_tokens_behind_a_block_of_scale_zero(top):
    """Older tokens whose scale is 0 are zeros whatever their codes are, and stay zeros."""
    t = torch()
    p = Paged([(3, 1)], 2, 64, 16, seed=26)
    bits, x = p.random_rows(2)
    x = (x / np.abs(x).max() * top).astype(np.float32)
    bits = WL.bf16_bits(x)
    for c in p.scale:
        c[p.blocks[0][0]] = 0.0
    LQ.kv_write(p.cache, p.batch(), to_dev(bits), to_dev(bits))
    LQ.get_device_status()
    K, V = (t.full((3, 2, 64), 0x7FC0, dtype=t.int16, device="cuda") for _ in range(2))
    LQ.kv_read(p.cache, p.batch([(3, 3)]), K, V)
    scale = np.abs(WL.bf16_to_f32(bits)).max(2)[0] / np.float32(127)
    for kv, got in enumerate((K, V)):
        v = bits_to_f32(got)
        assert (v[:2] == 0).all()
        assert np.array_equal(p.scale[kv][p.blocks[0][0]].cpu().numpy(), scale if top else np.ones(2, np.float32))
        assert (np.abs(v[2] - WL.bf16_to_f32(bits)[0]) <= 0.5001 * scale[:, None] + 2.0 ** -8 * np.abs(x[0])).all()


def _far(seqs_len, n, d, seed):
    """A sequence of `seqs_len` tokens whose blocks are one and the same but for its last six, and the short sequence
    of those six alone."""
    t = torch()
    width = -(-seqs_len // 128)
    p = Paged([(6 * 128 - (width * 128 - seqs_len), n)], 1, d, 128, seed=seed)
    table = t.full((1, width), p.blocks[0][0], dtype=t.int32, device="cuda")
    table[0, -6:] = t.tensor(p.blocks[0], dtype=t.int32)
    one = lambda v: t.tensor(v, dtype=t.int32, device="cuda")  # noqa: E731
    batch = lambda rows, max_rows: LQ.KVBatch.of(one([seqs_len]), one([0, rows]), table, rows, max_rows, seqs_len)  # noqa: E731
    return p, batch


LONGEST = (2 ** 31 - 1 - 1024) // 128 * 128               # the most that the host admits


@pytest.mark.parametrize("length,n,max_rows", [(LONGEST, 1, 1), (LONGEST - 3, 1, 2 ** 24), (LONGEST - 100, 200, 2 ** 20)])
def test_writes_and_reads_at_the_longest_lengths(length, n, max_rows):
    """The newest tokens of a sequence close to 2^31 tokens long, under bounds that allow many more rows than lie
    behind the last block."""
    t = torch()
    p, far = _far(length, n, 64, seed=27)
    _fill(p)
    before = [x.clone() for x in p.codes + p.scale]
    rows = [p.random_rows(1) for _ in range(2)]
    out = [[t.zeros((n, 1, 64), dtype=t.int16, device="cuda") for _ in range(2)] for _ in range(2)]
    after = []
    for batch, back in ((p.batch(), out[0]), (far(n, max_rows), out[1])):
        for x, start in zip(p.codes + p.scale, before):
            x.copy_(start)
        LQ.kv_write(p.cache, batch, to_dev(rows[0][0]), to_dev(rows[1][0]))
        LQ.kv_read(p.cache, batch, *back)
        LQ.get_device_status()
        after.append([x.nan_to_num() for x in p.codes + p.scale] + back)
    assert all(t.equal(a, b) for a, b in zip(*after)) and not t.equal(after[0][0], before[0])


@pytest.mark.parametrize("n", [1, 12, 40])
def test_windows_at_the_longest_lengths(n):
    p, far = _far(LONGEST - 3, n, 64, seed=28)
    vals = _fill(p)
    bits, q = p.random_rows(1)
    O = _attn(p, far(n, n), to_dev(bits), 0.2, 300, 1)
    LQ.get_device_status()
    _check(p, vals, O, q, 0.2, 300)


def test_attention_over_the_longest_length():
    """Every key of 2^31 - 1152 tokens, of which all but the last six blocks are one block over and over.  Bound: fp32
    sums of about 28,000 steps a warp and lane, each rounding once (2^-25 of the sum), in numerator and denominator."""
    p, far = _far(LONGEST - 3, 1, 64, seed=29)
    vals = _fill(p)
    bits, q = p.random_rows(1, scale=0.3)
    O = _attn(p, far(1, 1), to_dev(bits), 0.1, 0, 1)
    LQ.get_device_status()
    k, v = (x[:, 0] for x in vals[0])
    z = 0.1 * (k @ q[0, 0].astype(np.float64))
    w = np.exp(z - z.max())
    w[:128] *= LONGEST // 128 - 5                           # the repeated block stands at its own place too
    w /= w.sum()
    got, ref, mass = bits_to_f32(O)[0, 0], w @ v, w @ np.abs(v)
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2 * 28000 * 2.0 ** -25) * mass).all()
    assert np.abs(ref).max() > 4 * (2.0 ** -11 + 2 * 28000 * 2.0 ** -25) * mass.max()


def test_many_sequences_under_a_bound_far_above_their_lengths():
    """Thousands of sequences and heads with a length bound in the millions: the keys of one piece number no more than
    the bound, whatever the number of tiles."""
    t = torch()
    seqs, heads, width = 4096, 128, 78125
    p = Paged([(100, 1)], heads, 64, 128, seed=30)
    _fill(p)
    lens = (t.arange(seqs, device="cuda") % 101).int()
    start, table = t.arange(seqs + 1, device="cuda").int(), t.full((seqs, width), p.blocks[0][0], dtype=t.int32, device="cuda")
    Q = (t.randn(seqs, heads, 64, device="cuda") * 2).bfloat16()
    out = [_attn(p, LQ.KVBatch.of(lens, start, table, seqs, 1, bound), Q, 0.1, 0, heads, out=t.full_like(Q, float("nan")))
           for bound in (100, width * 128)]
    LQ.get_device_status()
    assert t.equal(*out) and (out[0][0] == 0).all() and (out[0][1:101].abs().amax((1, 2)) > 0).all()


@pytest.mark.parametrize("max_rows,max_len", [(0, 48), (2, 0), (0, 0)])
def test_bounds_of_zero_are_bounds(max_rows, max_len):
    """Sequences beyond bounds of zero rows or zero tokens are reported as beyond any other bound; what lies within
    them is served."""
    t = torch()
    p = Paged([(40, 2), (0, 1)], 2, 128, 16, seed=31)
    vals = _fill(p)
    del vals
    bits, _ = p.random_rows(2)
    K = to_dev(bits)
    batch = p.batch()
    batch.max_rows, batch.max_len = max_rows, max_len
    before = [c.clone() for c in p.codes]
    O = t.full((3, 2, 128), 1, dtype=t.int16, device="cuda")
    for call in (lambda: LQ.kv_write(p.cache, batch, K, K), lambda: LQ.kv_read(p.cache, batch, O, O),
                 lambda: _attn(p, batch, K, 0.1, 0, 2, out=O)):
        call()
        with pytest.raises(LQ.LrqatError) as e:
            LQ.get_device_status()
        assert e.value.status == -7
    assert all(t.equal(a, b) for a, b in zip(before, p.codes)) and (O[:2] == 1).all()
    assert (O[2] == (1 if max_rows == 0 else 0)).all()     # an idle slot's row, within the bounds or not


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("how", ["argument", "current"])
def test_calls_are_queued_behind_the_work_of_their_stream(how, new):
    """On a side stream some milliseconds of other work and then the copies that fill the inputs: a call on any other
    stream would read what the inputs or the cache held before."""
    t = torch()
    p = Paged([(90, new), (new, new)], 2, 128, 16, seed=32)
    _fill(p)
    src = [to_dev(p.random_rows(h)[0]) for h in (2, 2, 8)]
    start = [x.clone() for x in p.codes + p.scale]
    junk, side, batch = empty((1 << 28,), t.float32), t.cuda.Stream(), p.batch()

    def run(stream):
        for x, y in zip(p.codes + p.scale, start):
            x.copy_(y)
        K, V, Q = (t.zeros_like(x) for x in src)
        K2, V2, O = (t.zeros_like(x) for x in src)
        ws = empty((LQ.kv_attn_workspace_bytes(p.cache, batch, 8, 0),), t.uint8)
        other = stream or t.cuda.current_stream()
        other.wait_stream(t.cuda.current_stream())
        with t.cuda.stream(other):
            for i in range(20):
                junk.fill_(float(i))
            for x, y in zip((K, V, Q), src):
                x.copy_(y)
        with t.cuda.stream(stream if how == "current" else None):
            at = stream if how == "argument" else None
            LQ.kv_write(p.cache, batch, K, V, stream=at)
            LQ.kv_read(p.cache, batch, K2, V2, stream=at)
            LQ.kv_attn(p.cache, batch, Q, 0.1, 0, O, ws, stream=at)
        t.cuda.synchronize()
        return [x.nan_to_num() for x in p.codes + p.scale + [K2, V2, O]]

    assert all(t.equal(a, b) for a, b in zip(run(None), run(side)))


@pytest.mark.parametrize("scale", [-0.1, 0.0, -0.0])
@pytest.mark.parametrize("new", [1, 6, 100])
def test_softmax_scales_that_are_not_positive(new, scale):
    p = Paged([(333, new), (20, min(new, 20))], 2, 128, 16, seed=24)
    vals = _fill(p)
    bits, q = p.random_rows(4)
    O = _attn(p, p.batch(), to_dev(bits), scale, 0, 4)
    LQ.get_device_status()
    _check(p, vals, O, q, scale, 0)


def test_a_long_sequence_beside_a_prompt():
    """One new token of a long sequence in the batch of a prompt, whose tiles fill the machine: nothing is cut."""
    seqs = [(20000, 1), (1300, 1300)]
    p = Paged(seqs, 8, 64, 64, seed=25)
    vals = _fill(p)
    bits, q = p.random_rows(32)
    got = bits_to_f32(_attn(p, p.batch(), to_dev(bits), 0.1, 0, 32)).astype(np.float64)
    LQ.get_device_status()
    for b, rows, last in ((0, slice(0, 1), 20000), (1, slice(1, 4), 3), (1, slice(690, 700), 699), (1, slice(1297, 1301), 1300)):
        k, v = vals[b]
        ref, mass, seen = SO.attention(q[rows], k[:last], v[:last], last, 0.1)
        bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -11 * mass + (seen[:, None, None] * 2.0 ** -25) * np.abs(v).max()
        assert (np.abs(got[rows] - ref) <= bound).all()
