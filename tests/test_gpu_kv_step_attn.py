"""GPU parity of attention over the 8-bit cache through windows with sinks and over shared prefixes, against numpy.  The
tolerances are those of test_gpu_kv.py: both run its kernels, and joining one more part rounds in fp32."""
import numpy as np
import pytest

from oracle import serving_oracle as SO
from paper_2406_06385_gb300 import lrqat as LQ

from gpu_util import bits_to_f32, empty, to_dev, torch
from test_gpu_kv import LONGEST, Paged, _attn, _far, _fill, _seq_rows

pytestmark = pytest.mark.gpu


def _sinks(p, batch, Q, scale, window, sinks, n_heads, out=None, stream=None):
    t = torch()
    O = t.full(Q.shape, 0x7FC0, dtype=t.int16, device="cuda") if out is None else out
    ws = empty((LQ.kv_attn_sinks_workspace_bytes(p.cache, batch, n_heads, window, sinks),), t.uint8)
    ws.fill_(0xFF)
    LQ.kv_attn_sinks(p.cache, batch, Q, scale, window, sinks, O, ws, stream=stream)
    return O


def _bound(ref, mass, seen, top):
    return 2.0 ** -8 * np.abs(ref) + 2.0 ** -11 * mass + (seen[:, None, None] * 2.0 ** -25) * top


def _check(p, vals, O, q, scale, window=0, sinks=0, rows=None):
    got = bits_to_f32(O).astype(np.float64)
    for b, length, n, at in _seq_rows(p.seqs):
        some = np.arange(n) if rows is None else rows(n)
        for i in some if rows is not None else [None]:
            sl, end = (at, length) if i is None else (slice(at.start + i, at.start + i + 1), length - n + i + 1)
            ref, mass, seen = SO.attention(q[sl], *[v[:max(end, 0)] for v in vals[b]], end, scale, window, sinks)
            top = np.abs(vals[b][1]).max(initial=0.0)
            bad = ~(np.abs(got[sl] - ref) <= _bound(ref, mass, seen, top))
            assert not bad.any(), (b, i, np.argwhere(bad)[:5], got[sl][bad][:5], ref[bad][:5])


# ---------------------------------------------------------------------------- windows with sinks
SINKS = [
    # sequences (length, new), kv heads, group, d, block, window, sinks
    ([(1, 1)], 1, 1, 128, 16, 1, 1),
    ([(1, 1), (5, 1), (40, 1), (41, 1), (65, 1), (129, 1), (700, 1)], 2, 4, 128, 16, 8, 4),
    ([(1000, 1), (0, 1), (333, 1), (2049, 1)], 8, 4, 128, 64, 100, 4),
    ([(3000, 1), (90, 1)], 5, 1, 64, 32, 33, 70),
    ([(300, 1), (31, 1)], 1, 16, 64, 128, 17, 1),
    ([(300, 2), (131, 1)], 2, 7, 128, 16, 50, 33),
    ([(300, 2), (131, 1)], 2, 7, 128, 16, 1, 64),
    ([(130, 3), (264, 1)], 1, 71, 128, 16, 64, 4),
    ([(500, 200), (333, 300), (40, 40)], 1, 2, 64, 16, 64, 5),
    ([(900, 64), (1500, 3)], 2, 8, 128, 64, 511, 100),
    ([(1500, 300)], 2, 4, 128, 16, 129, 16),
    ([(1500, 300)], 1, 4, 128, 128, 1, 65),
    ([(1200, 40)], 2, 4, 64, 32, 700, 200),
    ([(3, 9), (120, 21), (0, 4), (250, 2)], 2, 4, 128, 16, 10, 3),        # padding rows before the first position
    ([(20000, 1)], 1, 8, 128, 128, 6000, 4),
    ([(9000, 4)], 2, 1, 128, 16, 3000, 130),
    ([(9000, 30)], 1, 4, 64, 16, 2500, 1000),
]


@pytest.mark.parametrize("seqs,heads,group,d,block,window,sinks", SINKS)
def test_sinks(seqs, heads, group, d, block, window, sinks):
    """Blocks that no row sees have table entries outside the pool: they are not followed."""
    t = torch()
    p = Paged(seqs, heads, d, block, seed=len(seqs) + block + sinks)
    vals = _fill(p)
    for b, (length, n) in enumerate(seqs):
        first = max(0, max(0, length - n) - window + 1)
        for c in range(-(-sinks // block), first // block):
            p.table[b, c] = -5
    bits, q = p.random_rows(heads * group)
    scale = 1.3 / np.sqrt(d)
    O = _sinks(p, p.batch(), to_dev(bits), scale, window, sinks, heads * group)
    LQ.get_device_status()
    _check(p, vals, O, q, scale, window, sinks)
    assert t.equal(O, _sinks(p, p.batch(), to_dev(bits), scale, window, sinks, heads * group))
    loose = p.batch(slack=200)                               # larger bounds cut the keys otherwise
    _check(p, vals, _sinks(p, loose, to_dev(bits), scale, window, sinks, heads * group), q, scale, window, sinks)
    LQ.get_device_status()


@pytest.mark.parametrize("new", [1, 3, 40])
def test_no_sinks_and_windows_that_hide_nothing(new):
    t = torch()
    p = Paged([(500, new), (77, new)], 2, 128, 16, seed=16)
    vals = _fill(p)
    bits, q = p.random_rows(8)
    Q = to_dev(bits)
    for window in (0, 1, 100, 2 ** 31 - 1):
        assert t.equal(_sinks(p, p.batch(), Q, 0.1, window, 0, 8), _attn(p, p.batch(), Q, 0.1, window, 8))
    whole = _attn(p, p.batch(), Q, 0.1, 0, 8)
    for window, sinks in ((0, 4), (0, 2 ** 31 - 1), (100, 400), (1, 499), (1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert t.equal(_sinks(p, p.batch(), Q, 0.1, window, sinks, 8), whole)
    for window, sinks in ((1, 498), (100, 399), (495, 4)):   # one key hidden from the last row
        _check(p, vals, _sinks(p, p.batch(), Q, 0.1, window, sinks, 8), q, 0.1, window, sinks)
    LQ.get_device_status()


@pytest.mark.parametrize("new", [1, 6, 100])
def test_what_lies_between_sinks_and_window_does_not_leak(new):
    """NaN scales in the blocks between; a NaN scale among the sinks reaches every row."""
    window, length, sinks = 48, 600, 20
    p = Paged([(length, new)], 2, 128, 16, seed=10)
    vals = _fill(p)
    first = max(0, length - new - window + 1)
    for kv in range(2):
        for i in range(2, first // 16):
            p.scale[kv][p.blocks[0][i]] = float("nan")
    bits, q = p.random_rows(4)
    O = _sinks(p, p.batch(), to_dev(bits), 0.1, window, sinks, 4)
    LQ.get_device_status()
    _check(p, vals, O, q, 0.1, window, sinks)
    p.scale[0][p.blocks[0][1]] = float("nan")
    assert np.isnan(bits_to_f32(_sinks(p, p.batch(), to_dev(bits), 0.1, window, sinks, 4))).all()
    assert not np.isnan(bits_to_f32(_sinks(p, p.batch(), to_dev(bits), 0.1, window, 16, 4))).any()


@pytest.mark.parametrize("n", [1, 12, 40])
def test_sinks_at_the_longest_lengths(n):
    """The sequence's first tokens are those of its repeated block, 2^31 tokens before its window."""
    p, far = _far(LONGEST - 3, n, 64, seed=28)
    vals = _fill(p)
    bits, q = p.random_rows(1)
    O = _sinks(p, far(n, n), to_dev(bits), 0.2, 300, 40, 1)
    LQ.get_device_status()
    _check(p, vals, O, q, 0.2, 300, 40)                      # the short sequence starts with the same block


@pytest.mark.parametrize("scale", [-0.1, 0.0])
@pytest.mark.parametrize("new", [1, 6, 100])
def test_sinks_with_scales_that_are_not_positive_and_zero_values(new, scale):
    def zeros(kv, used, s):
        if kv == 1:
            s[::3] = 0.0
        return s

    p = Paged([(433, new), (220, min(new, 20))], 2, 128, 16, seed=24)
    vals = _fill(p, zeros)
    bits, q = p.random_rows(4)
    O = _sinks(p, p.batch(), to_dev(bits), scale, 60, 7, 4)
    LQ.get_device_status()
    _check(p, vals, O, q, scale, 60, 7)


# ---------------------------------------------------------------------------- shared prefixes
class Shared(Paged):
    """Sequences whose first `prefix` tokens lie in common blocks."""

    def __init__(self, prefix, own, heads, d, block, seed=0, kv_scale=None):
        """own: (tokens behind the prefix, new rows); a first number below 0 is a whole length inside the prefix,
        -1 - length."""
        seqs = [(prefix + m if m >= 0 else -1 - m, n) for m, n in own]
        super().__init__([(prefix, 0)] + [(max(0, length - prefix), n) for length, n in seqs], heads, d, block, seed)
        vals = _fill(self, kv_scale)
        first = prefix // block
        self.prefix, self.prefix_blocks = prefix, self.blocks[0]
        table, self.blocks = self.table, [self.blocks[0] + bl for bl in self.blocks[1:]]
        self.table = np.full((len(seqs), first + max(1, table.shape[1])), -7, np.int32)    # no column of the prefix is followed
        self.table[:, first:first + table.shape[1]] = table[1:]
        self.seqs = seqs
        self.vals = [[np.concatenate([a, b])[:length] for a, b in zip(vals[0], v)] for v, (length, _) in zip(vals[1:], seqs)]
        self.together = None
        self.prefix_table = to_dev(np.array(self.prefix_blocks, np.int32))

    def attend(self, Q, scale, n_heads, batch=None, out=None, stream=None):
        t = torch()
        batch = self.batch() if batch is None else batch
        O = t.full(Q.shape, 0x7FC0, dtype=t.int16, device="cuda") if out is None else out
        ws = empty((LQ.kv_attn_shared_workspace_bytes(self.cache, batch, n_heads, self.prefix),), t.uint8)
        ws.fill_(0xFF)
        LQ.trace_enable(True)
        LQ.kv_attn_shared(self.cache, batch, self.prefix_table, self.prefix, Q, scale, O, ws, stream=stream)
        LQ.trace_enable(False)
        launches = LQ.trace_read()["kv_attn_shared"][0]
        if self.together is not None:                        # over the prefix, over the own keys, the join
            assert (launches == 3) == self.together
        return O


SHARED = [
    # prefix, own tokens and new rows, kv heads, group, d, block
    (16, [(1, 1)], 1, 1, 128, 16),
    (16, [(1, 1), (3, 1)], 1, 1, 128, 16),
    (48, [(1, 1), (20, 1), (33, 1)], 2, 2, 64, 16),
    (1040, [(61, 1), (61, 1)], 8, 4, 128, 16),
    (640, [(1, 1), (1000, 1), (17, 1), (-1, 1), (129, 1)], 2, 4, 128, 128),       # an idle slot
    (320, [(5, 5), (40, 3), (9, 2)], 3, 1, 128, 64),
    (96, [(5, 5), (40, 3), (0, 0), (9, 2)], 1, 71, 128, 32),
    (2000, [(i % 7 + 1, 1) for i in range(40)], 2, 4, 128, 16),
    (4096, [(i * 13 + 1, 1) for i in range(70)], 1, 8, 64, 64),
    (144, [(1, 1)] * 3 + [(-1 - 100, 1), (-1 - 16, 9), (-1 - 144, 3)], 2, 2, 128, 16),   # sequences inside the prefix
    (144, [(2, 9), (-1 - 5, 9), (-1, 4)], 2, 4, 128, 16),                         # rows at both sides, padding rows
    (256, [(300, 300), (77, 50)], 2, 4, 128, 64),
    (48, [(200, 33), (64, 64), (-1 - 40, 37)], 1, 8, 64, 16),
    (512, [(600, 1)], 4, 8, 128, 128),
    (16, [(3000, 1), (2500, 1), (1, 1)], 4, 2, 128, 16),
    (20000, [(7, 2), (300, 1)], 2, 4, 128, 32),
    (3104, [(10, 20), (15, 18), (3, 3)], 2, 4, 64, 16),
    (640, [(2, 30), (-1 - 5, 30), (-1, 4), (-1 - 100, 25), (0, 0), (300, 1)], 2, 4, 128, 128),
    (512, [(i, 17) for i in range(9)], 3, 1, 64, 16),
    (576, [(130, 1), (7, 2)], 1, 60, 128, 64),
]
# where the prefix is read once for all: in 8-row tiles, in one and two 16-row tiles, in 256-row tiles; the own keys in
# tiles of 8, 16 and 256 rows; with padding, sequences inside the prefix and rows at both sides of its end
TOGETHER = [
    (16000, [(1, 1), (20, 1)], 8, 4, 128, 64),
    (12800, [(1, 1), (20, 1)], 20, 4, 128, 16),
    (16000, [(1, 1), (20, 1), (-1 - 100, 1), (-1, 1)], 8, 4, 128, 16),
    (16000, [(3, 1)] * 5 + [(-1 - 7000, 1), (-1 - 64, 1), (200, 1)], 8, 4, 128, 64),
    (8000, [(3, 1)] * 9 + [(-1 - 7000, 1), (-1 - 64, 1), (200, 1)], 8, 4, 64, 64),
    (4096, [(i * 13 % 70 + 1, 1) for i in range(37)] + [(-1, 1), (-1 - 4000, 1), (-1 - 64, 1)], 8, 4, 64, 64),
    (4096, [(5, 4), (40, 3), (9, 2), (-1 - 2, 4), (-1 - 1599, 1), (1, 4), (-1 - 4096, 2), (60, 4), (5, 4), (7, 4)], 8, 4, 128, 32),
    (4096, [(2, 8), (-1 - 5, 8), (-1, 4), (-1 - 100, 8), (0, 0), (300, 1), (8, 8)], 8, 4, 128, 128),
    (2000, [(9, 5)] * 14 + [(1, 5), (-1 - 3, 5)], 40, 1, 128, 16),
    (16000, [(2000, 32), (1500, 20), (3, 7)], 8, 4, 128, 64),
    (16000, [(3, 4), (90, 1), (4, 4)], 8, 30, 64, 32),
]


@pytest.mark.parametrize("prefix,own,heads,group,d,block,together",
                         [c + (False,) for c in SHARED] + [c + (True,) for c in TOGETHER])
def test_shared(prefix, own, heads, group, d, block, together):
    t = torch()
    p = Shared(prefix, own, heads, d, block, seed=prefix + len(own))
    p.together = together
    bits, q = p.random_rows(heads * group)
    scale = 1.3 / np.sqrt(d)
    O = p.attend(to_dev(bits), scale, heads * group)
    LQ.get_device_status()
    some = (lambda n: sorted({0, n - 1}) if n else []) if together else None
    _check(p, p.vals, O, q, scale, rows=some)
    assert t.equal(O, p.attend(to_dev(bits), scale, heads * group))
    slack = min(200, p.table.shape[1] * block - max(n for n, _ in p.seqs))
    loose = p.batch(slack=slack)
    if together:                                             # with bounds for which it still is
        loose.max_rows = p.batch().max_rows
        if len(bits) * group <= 8:
            p.together = None                                # but for the tiles that three rows more need
    behind = 3 if together else 50                           # rows behind the last sequence: left as they were
    loose.rows += behind
    wide = t.full((len(bits) + behind,) + bits.shape[1:], 7, dtype=t.int16, device="cuda")
    Q = t.zeros_like(wide)
    Q[:len(bits)] = to_dev(bits)
    p.attend(Q, scale, heads * group, loose, out=wide)
    LQ.get_device_status()
    _check(p, p.vals, wide[:len(bits)], q, scale, rows=some)
    assert (wide[len(bits):] == 7).all()


@pytest.mark.parametrize("new", [1, 4, 40])
def test_no_prefix_is_the_plain_call(new):
    t = torch()
    p = Paged([(500, new), (77, new)], 2, 128, 16, seed=16)
    _fill(p)
    Q = to_dev(p.random_rows(8)[0])
    out = t.zeros_like(Q)
    batch = p.batch()
    ws = empty((LQ.kv_attn_shared_workspace_bytes(p.cache, batch, 8, 0),), t.uint8)
    LQ.kv_attn_shared(p.cache, batch, None, 0, Q, 0.1, out, ws)
    assert t.equal(out, _attn(p, batch, Q, 0.1, 0, 8))


@pytest.mark.parametrize("own,prefix,heads", [
    ([(30, 1), (200, 1), (1, 1)], 160, 2), ([(30, 6), (200, 6), (7, 6)], 160, 2), ([(300, 100), (100, 100)], 160, 2),
    ([(30, 1), (200, 1), (1, 1)], 16000, 8), ([(30, 6), (200, 6), (7, 6), (50, 6)], 16000, 8), ([(300, 20), (100, 17)], 20000, 8)])
def test_shared_scales_far_apart_and_zero(own, prefix, heads):
    """Values of 1e20 behind negligible weights, tiny ones behind the whole weight, blocks of scale 0; on either side of the
    prefix's end.  Bound as for one table."""
    def far(kv, used, scale):
        if kv == 1:
            scale = (10.0 ** rng.uniform(-20, 20, scale.shape)).astype(np.float32)
            scale[::5] = 0.0
        return scale

    rng = np.random.default_rng(3)
    p = Shared(prefix, own, heads, 128, 16, seed=8, kv_scale=far)
    p.together = prefix > 160
    bits, q = p.random_rows(2 * heads)
    O = p.attend(to_dev(bits), 0.5, 2 * heads)
    LQ.get_device_status()
    got = bits_to_f32(O).astype(np.float64)
    for b, length, n, at in _seq_rows(p.seqs):
        ref, mass, seen = SO.attention(q[at], *p.vals[b], length, 0.5)
        z = 0.5 * np.abs(np.einsum("nhd,lhd->nhl", q[at].astype(np.float64), np.repeat(p.vals[b][0], 2, 1))).max()
        bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + (z + 100) * 2.0 ** -21 + seen[:, None, None] * 2.0 ** -18) * mass.max(2, keepdims=True)
        assert (np.abs(got[at] - ref) <= bound).all()


@pytest.mark.parametrize("new,prefix,heads", [(1, 160, 2), (6, 160, 2), (100, 160, 2), (1, 20000, 8), (20, 20000, 8), (40, 20000, 8)])
def test_nan_in_one_sequence_stays_there(new, prefix, heads):
    p = Shared(prefix, [(200, new), (150, new)], heads, 128, 16, seed=9)
    p.together = prefix > 160
    bits, q = p.random_rows(2 * heads)
    ref = bits_to_f32(p.attend(to_dev(bits), 0.1, 2 * heads))
    p.scale[1][p.blocks[1][-1]] = float("nan")
    bad = bits.copy()
    bad[0, 1, 5] = 0x7FC0
    got = bits_to_f32(p.attend(to_dev(bad), 0.1, 2 * heads))
    assert np.isnan(got[0, 1]).all() and np.isnan(got[-1]).all()
    hit = np.zeros(got.shape[:2], bool)
    hit[0, 1] = True
    hit[new:] = True                                         # rows of the other sequence may see its last block
    # which rows look for a new maximum is decided for 32 rows at a time, so the others agree within rounding
    assert (np.abs(got[~hit] - ref[~hit]) <= 2.0 ** -7 * np.abs(ref[~hit]) + 2.0 ** -10 * np.abs(p.vals[0][1]).max()).all()


@pytest.mark.parametrize("own,prefix,heads", [([(30, 1), (200, 1), (1, 1)], 160, 2), ([(300, 100), (100, 100)], 160, 2),
                                              ([(30, 1), (200, 1), (1, 1)], 16000, 8), ([(30, 5), (200, 6), (7, 4), (9, 6)], 16000, 8),
                                              ([(300, 20), (100, 17)], 20000, 8)])
def test_shared_bounds_and_bad_blocks_are_reported(own, prefix, heads):
    """A sequence beyond the batch's bounds, or with a block outside the pool, is reported, and the others are served; so is
    a block of the prefix outside the pool."""
    t = torch()
    p = Shared(prefix, own, heads, 128, 16, seed=14)
    p.together = prefix > 160
    bits, q = p.random_rows(2 * heads)
    Q = to_dev(bits)
    n0 = own[0][1]

    def expect(batch):
        O = p.attend(Q, 0.1, 2 * heads, batch)
        with pytest.raises(LQ.LrqatError) as e:
            LQ.get_device_status()
        assert e.value.status == -7
        LQ.get_device_status()
        got = bits_to_f32(O).astype(np.float64)
        for b, length, n, at in _seq_rows(p.seqs):
            if b:
                at = slice(at.stop - min(n, 3 if p.together else n), at.stop)
                ref, mass, seen = SO.attention(q[at], *p.vals[b], length, 0.1)
                assert (np.abs(got[at] - ref) <= _bound(ref, mass, seen, np.abs(p.vals[b][1]).max())).all()
        return O

    for what, value in (("table", p.cache.n_blocks), ("table", -1), ("lens", 10 ** 6), ("lens", -5)):
        batch = p.batch()
        if what == "lens":
            batch.tensors[0][0] = value
        else:
            batch.tensors[2][0, :] = value
        O = expect(batch)
        if what == "lens":
            assert (O[:n0] == 0x7FC0).all()                  # skipped
    batch = p.batch()
    batch.tensors[1][0] = -1                                 # its rows start before the batch's
    expect(batch)
    p.prefix_table[3] = 10 ** 6
    p.attend(Q, 0.1, 2 * heads)
    with pytest.raises(LQ.LrqatError) as e:
        LQ.get_device_status()
    assert e.value.status == -7


@pytest.mark.parametrize("own,group,prefix,kv_heads", [
    ([(31, 1)] * 3, 4, 320, 2), ([(31, 1)] * 9, 4, 320, 2), ([(31, 5)] * 9, 4, 320, 2), ([(90, 90)] * 2, 4, 320, 2),
    ([(31, 1)] * 9, 4, 8000, 8), ([(31, 4)] * 9, 4, 4800, 8), ([(31, 8)] * 5, 4, 4800, 8)])
def test_shared_strided_rows_other_streams_and_graphs(own, group, prefix, kv_heads):
    """Q and O as parts of wider rows, on a side stream; a captured call replayed for other lengths, for another number of
    rows, and beside a second graph with a workspace of its own."""
    t = torch()
    p = Shared(prefix, [(m + 40, n) for m, n in own], kv_heads, 128, 16, seed=12)
    p.together = prefix > 320
    vals = p.vals
    p.seqs = [(prefix + m, n) for m, n in own]
    heads, rows = kv_heads * group, sum(n for _, n in own)
    bits, q = p.random_rows(heads)
    batch = p.batch(slack=40)
    if p.together:                                           # with bounds for which it still is
        batch.max_rows = own[0][1]
    ref = p.attend(to_dev(bits), 0.1, heads, batch)
    wide = t.zeros((rows, heads + 8, 128), dtype=t.int16, device="cuda")
    wide[:, 4:4 + heads] = to_dev(bits)
    out = t.zeros((rows, heads + 12, 128), dtype=t.int16, device="cuda")
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        p.attend(wide[:, 4:4 + heads], 0.1, heads, batch, out=out[:, 8:8 + heads])
    side.synchronize()
    assert t.equal(out[:, 8:8 + heads], ref) and (out[:, :8] == 0).all() and (out[:, 8 + heads:] == 0).all()
    lens, Q = batch.tensors[0], to_dev(bits)
    outs, graphs = [t.zeros_like(Q) for _ in range(2)], []
    for O in outs:
        ws = empty((LQ.kv_attn_shared_workspace_bytes(p.cache, batch, heads, prefix),), t.uint8)
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            LQ.kv_attn_shared(p.cache, batch, p.prefix_table, prefix, Q, 0.1, O, ws)
        graphs.append((graph, ws))
    for add in (0, 37, -25, -320):
        lens.copy_(t.tensor([prefix + m + add for m, _ in own], dtype=t.int32))
        streams = [t.cuda.Stream() for _ in graphs]
        for s, (graph, _) in zip(streams, graphs):
            s.wait_stream(t.cuda.current_stream())
            with t.cuda.stream(s):
                graph.replay()
        t.cuda.synchronize()
        p.seqs = [(prefix + m + add, n) for m, n in own]
        cut = [[v[:prefix + m + add] for v in vs] for vs, (m, _) in zip(vals, own)]
        assert t.equal(*outs)
        _check(p, cut, outs[0], q, 0.1, rows=(lambda n: sorted({0, n - 1})) if p.together else None)


@pytest.mark.parametrize("own,prefix", [([(1, 1)] * 2, 30000), ([(60, 1)] * 64, 6000), ([(300, 1)] * 20, 640),
                                        ([(300, 4)] * 20, 640), ([(9, 5)] * 16, 2000)])
def test_shared_results_do_not_depend_on_where_the_cache_lies(own, prefix):
    t = torch()
    p = Shared(prefix, own, 8, 128, 16, seed=15)
    bits, q = p.random_rows(32)
    Q, batch = to_dev(bits), p.batch()
    junk = t.empty(1 << 28, dtype=t.float32, device="cuda")
    out = []
    for i in range(6):
        if i < 4:
            junk.fill_(float(i))
        out.append(p.attend(Q, 0.1, 32, batch))
    LQ.get_device_status()
    assert all(t.equal(o, out[0]) for o in out)
    p.seqs, q, keep = p.seqs[-2:], q[-2 * own[0][1]:], out[0][-2 * own[0][1]:]
    _check(p, p.vals[-2:], keep, q, 0.1, rows=lambda n: [n - 1])


@pytest.mark.parametrize("window,sinks", [(0, 0), (8, 4)])
def test_tiles_of_padding_alone(window, sinks):
    """Tiles of 256 rows none of which has a position, next to some that have: rows of zeros, call after call."""
    t = torch()
    p = Paged([(0, 300), (40, 300), (0, 65), (70, 70)], 2, 128, 16)
    vals = _fill(p)
    bits, q = p.random_rows(8)
    Q, batch = to_dev(bits), p.batch()
    first = _sinks(p, batch, Q, 0.1, window, sinks, 8)
    _check(p, vals, first, q, 0.1, window, sinks)
    for _ in range(20):
        assert t.equal(_sinks(p, batch, Q, 0.1, window, sinks, 8), first)


@pytest.mark.parametrize("call,new,prefix,heads", [("sinks", 1, 160, 2), ("sinks", 40, 160, 2), ("shared", 1, 160, 2),
                                                   ("shared", 40, 160, 2), ("shared", 1, 20000, 8), ("shared", 10, 20000, 8)])
def test_calls_are_queued_behind_the_work_of_their_stream(call, new, prefix, heads):
    t = torch()
    p = Shared(prefix, [(90, new), (new, new)], heads, 128, 16, seed=32)
    p.table[:, :prefix // 16] = np.array(p.prefix_blocks)
    src = to_dev(p.random_rows(4 * heads)[0])
    junk, side, batch = empty((1 << 28,), t.float32), t.cuda.Stream(), p.batch()

    def run(stream):
        Q, O = t.zeros_like(src), t.zeros_like(src)
        other = stream or t.cuda.current_stream()
        other.wait_stream(t.cuda.current_stream())
        with t.cuda.stream(other):
            for i in range(20):
                junk.fill_(float(i))
            Q.copy_(src)
        size = (LQ.kv_attn_sinks_workspace_bytes(p.cache, batch, 4 * heads, 30, 5) if call == "sinks"
                else LQ.kv_attn_shared_workspace_bytes(p.cache, batch, 4 * heads, prefix))
        ws = empty((size,), t.uint8)
        if call == "sinks":
            LQ.kv_attn_sinks(p.cache, batch, Q, 0.1, 30, 5, O, ws, stream=stream)
        else:
            LQ.kv_attn_shared(p.cache, batch, p.prefix_table, prefix, Q, 0.1, O, ws, stream=stream)
        t.cuda.synchronize()
        return O

    assert t.equal(run(None), run(side))
