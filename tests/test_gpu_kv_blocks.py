"""Cache blocks handed out and taken back on the device, against the sequential definition: everything is whole numbers and
has to be equal."""
import numpy as np
import pytest

from oracle import serving_oracle as SO
from paper_2406_06385_gb300 import lrqat as LQ

from gpu_util import empty, to_dev, torch

pytestmark = pytest.mark.gpu


class Pool:
    """Device and oracle state side by side."""

    def __init__(self, n_seqs, max_blocks, capacity, free, block, pinned=0, seed=0, length=None):
        t = torch()
        rng = np.random.default_rng(seed)
        ids = rng.permutation(capacity).astype(np.int32)
        table = rng.integers(10 ** 6, 10 ** 7, (n_seqs, max_blocks)).astype(np.int32)      # what nobody may follow
        length = np.zeros(n_seqs, np.int32) if length is None else np.asarray(length, np.int32)
        ids[free:] = -9
        self.ref = SO.Blocks(table, ids, free, length, block, pinned)
        self.table, self.ids, self.len = to_dev(table), to_dev(ids), to_dev(length)
        self.free = t.tensor([free], dtype=t.int32, device="cuda")
        self.blocks = LQ.KVBlocks.of(self.table, self.ids, block, pinned)
        self.ws = empty((LQ.kv_blocks_workspace_bytes(self.blocks),), t.uint8)
        self.n = n_seqs

    def extend(self, add, slack=0, refused=False, rows=None, in_place=True, slots=True):
        t = torch()
        rows = int(np.abs(np.asarray(add, np.int64)).sum()) + slack if rows is None else rows
        full = lambda n, dt=t.int32: t.full((n,), -77, dtype=dt, device="cuda")  # noqa: E731
        seen, start, pos, slot = full(self.n), full(self.n + 1), full(rows), full(rows, t.int64)
        len_out, free_out = (self.len, self.free) if in_place else (full(self.n), full(1))
        self.ws.fill_(0xFF)
        LQ.kv_extend(self.blocks, self.len, to_dev(np.asarray(add, np.int32)), self.free, len_out, free_out, seen, start,
                     pos, slot if slots else None, self.ws)
        self._status(refused)
        self.len, self.free = len_out, free_out
        want = self.ref.extend(add, rows)
        assert want[4] == refused
        for got, ref in zip((seen, start, pos, slot), want):
            if got is not slot or slots:
                assert np.array_equal(got.cpu().numpy(), np.asarray(ref, np.int64)), (got, ref)
        self._same()
        return seen, start, pos, slot

    def truncate(self, keep, refused=False, in_place=True):
        t = torch()
        len_out, free_out = (self.len, self.free) if in_place else (t.zeros_like(self.len), t.zeros_like(self.free))
        LQ.kv_truncate(self.blocks, self.len, to_dev(np.asarray(keep, np.int32)), self.free, len_out, free_out, self.ws)
        self._status(refused)
        self.len, self.free = len_out, free_out
        assert self.ref.truncate(keep) == refused
        self._same()

    def _status(self, refused):
        if refused:
            with pytest.raises(LQ.LrqatError) as e:
                LQ.get_device_status()
            assert e.value.status == -7
        LQ.get_device_status()

    def _same(self):
        assert np.array_equal(self.len.cpu().numpy(), self.ref.len)
        assert int(self.free) == self.ref.free
        assert np.array_equal(self.table.cpu().numpy(), self.ref.table)
        assert np.array_equal(self.ids.cpu().numpy(), self.ref.free_ids)


@pytest.mark.parametrize("n_seqs,block,pinned,top", [
    (1, 16, 0, 40), (3, 16, 0, 1), (3, 128, 2, 300), (31, 32, 0, 70), (48, 16, 3, 1), (130, 16, 0, 9), (1023, 16, 0, 3),
    (1024, 64, 1, 2), (1025, 16, 0, 5), (2100, 32, 0, 40), (20, 16, 0, 3000)])
def test_running_sequences(n_seqs, block, pinned, top):
    """Steps of new tokens, paused and idle slots and padding, shortened and finished sequences, in place and not."""
    rng = np.random.default_rng(n_seqs + block)
    width = pinned + 4 * top // block + 4
    p = Pool(n_seqs, width, n_seqs * width + 5, n_seqs * width, block, pinned, seed=n_seqs)
    for turn in range(5):
        add = rng.integers(0, top + 1, n_seqs)
        add[rng.random(n_seqs) < 0.2] = 0
        idle = rng.random(n_seqs) < 0.1
        add[idle] = -rng.integers(1, 3, int(idle.sum()))
        room = width * block - np.asarray(p.ref.len)
        add = np.minimum(add, room)
        p.extend(add, slack=(0, 1, 37)[turn % 3], in_place=turn % 2 == 0, slots=turn != 3)
        keep = np.asarray(p.ref.len) - rng.integers(-2, top + 1, n_seqs)
        keep[rng.random(n_seqs) < 0.3] = -1
        if turn != 1:
            p.truncate(keep, in_place=turn % 2 == 1)
    p.truncate(np.zeros(n_seqs))
    assert int(p.free) == n_seqs * width


def test_blocks_given_back_are_handed_out_again():
    """Extending and taking all of it back leaves the list as it was, and a second call hands out the same blocks."""
    t = torch()
    p = Pool(200, 30, 6000, 5990, 16)
    p.extend(np.full(200, 33))
    before = (p.len.cpu().numpy().copy(), p.ids.clone(), int(p.free))
    p.extend(np.arange(200) % 50)
    table = p.table.clone()
    p.truncate(before[0])
    assert int(p.free) == before[2] and t.equal(p.ids, before[1])
    p.extend(np.arange(200) % 50)
    assert t.equal(p.table, table)


@pytest.mark.parametrize("rows", [None, 20000])
def test_requests_that_cannot_be_met(rows):
    """The list runs dry in the middle of the batch; sequences too long for their table, with impossible lengths, or behind
    the last row: they take nothing and are reported, the others are served."""
    p = Pool(6, 8, 64, 5, 16, length=[0, 3, 0, 0, 5, 0])
    p.extend([30, 40, 17, 50, 3, 1], refused=True, rows=rows)             # 2, then 2 of 3 left, 2 do not fit; 3 fits (0)
    p = Pool(4, 2, 64, 64, 16, length=[32, 20, 0, 40])
    p.extend([1, 12, 33, 0], refused=True, rows=rows)
    p = Pool(4, 2, 64, 64, 16, length=[0, -3, 0, 0])
    p.extend([1, 1, 2 ** 31 - 1, -2 ** 31], refused=True, rows=rows or 5)
    p = Pool(3, 2, 64, 64, 16)
    p.extend([4, 5, 1], refused=True, rows=8)
    for free in (-1, 65):
        p = Pool(3, 2, 64, 64, 16, length=[16, 3, 0])
        p.free.fill_(free)
        p.ref.free = free
        p.extend([1, 2, -1], refused=True, rows=rows)


def test_truncations_that_cannot_be_met():
    p = Pool(4, 4, 10, 6, 16, length=[64, 65, 20, 64])
    p.table[:] = to_dev(np.arange(16, dtype=np.int32).reshape(4, 4))
    p.ref.table[:] = np.arange(16).reshape(4, 4)
    p.truncate([16, 0, 16, 0], refused=True)                  # 3 come back; 65 tokens do not fit; 1; 4 more do not fit
    for free in (-1, 11):
        p = Pool(2, 4, 10, 6, 16, length=[64, 3])
        p.free.fill_(free)
        p.ref.free = free
        p.truncate([0, 3], refused=True)


@pytest.mark.parametrize("n_seqs", [1, 65535])
def test_the_most_sequences(n_seqs):
    rng = np.random.default_rng(9)
    p = Pool(n_seqs, 3, 3 * n_seqs, 3 * n_seqs, 16, seed=9)
    p.extend(rng.integers(-1, 20, n_seqs))
    p.extend(rng.integers(-1, 5, n_seqs))
    p.truncate(rng.integers(-1, 30, n_seqs))


@pytest.mark.parametrize("n_seqs", [3, 1024, 1025, 65535])
def test_steps_without_rows(n_seqs):
    """Every sequence pauses: lengths and row starts are laid out all the same, in one launch.  What then asks for rows does
    not fit them."""
    length = np.random.default_rng(n_seqs).integers(0, 33, n_seqs)
    p = Pool(n_seqs, 3, 16, 16, 16, length=length)
    LQ.trace_enable()
    try:
        seen, start, _, _ = p.extend(np.zeros(n_seqs, np.int32), rows=0, in_place=False)
        assert LQ.trace_read()["kv_extend"][0] == 1
    finally:
        LQ.trace_enable(False)
    assert np.array_equal(seen.cpu().numpy(), length) and not start.any()
    add = np.zeros(n_seqs, np.int32)
    add[-1] = 1
    p.extend(add, rows=0, refused=True)
    p.extend(np.zeros(n_seqs, np.int32), rows=0)
    p.extend(add, slots=False)
    p.truncate(length)


def test_long_rows_of_the_table():
    """One sequence of 2^31 - 1152 tokens takes its last blocks."""
    most = (2 ** 31 - 1 - 1024) // 128
    p = Pool(1, most, 10, 10, 128, length=[most * 128 - 300])
    p.extend([300])
    p.truncate([most * 128 - 256])


def test_captured_steps():
    """A captured step (extension in place, shortening in place) replayed with other requests; the batch it lays out drives
    the cache's own operators."""
    t = torch()
    p = Pool(5, 20, 200, 190, 16, seed=3)
    heads, d = 2, 64
    codes = [t.zeros((200, heads, 16, d), dtype=t.int8, device="cuda") for _ in range(2)]
    scale = [t.zeros((200, heads), device="cuda") for _ in range(2)]
    cache = LQ.KVCache.of(*codes, *scale)
    add, seen, start = (t.zeros(n, dtype=t.int32, device="cuda") for n in (5, 5, 6))
    rows = 64
    pos, slot = t.zeros(rows, dtype=t.int32, device="cuda"), t.zeros(rows, dtype=t.int64, device="cuda")
    batch = LQ.KVBatch.of(seen, start, p.table, rows, rows, 320)
    K, V = (t.zeros((rows, heads, d), dtype=t.bfloat16, device="cuda") for _ in range(2))

    def step():
        LQ.kv_extend(p.blocks, p.len, add, p.free, p.len, p.free, seen, start, pos, slot, p.ws)
        LQ.kv_write(cache, batch, K, V)

    step()                                                    # lengths stay 0: nothing is asked for
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        step()
    rng = np.random.default_rng(4)
    for turn in range(6):
        a = rng.integers(-1, 12, 5)
        add.copy_(t.tensor(a.tolist(), dtype=t.int32))
        k = t.randn(rows, heads, d, device="cuda").bfloat16()
        K.copy_(k)
        V.copy_(-k)
        graph.replay()
        LQ.get_device_status()
        want = p.ref.extend(a, rows)
        for got, ref in zip((seen, start, pos, slot), want):
            assert np.array_equal(got.cpu().numpy(), np.asarray(ref, np.int64))
        p._same()
        # the new rows lie where their slots say
        live = (slot >= 0).nonzero().flatten()
        got = codes[0].transpose(1, 2).reshape(-1, heads, d)[slot[live]].float()
        s = scale[0][slot[live] // 16][..., None]
        assert ((got * s - k[live].float()).abs() <= 0.51 * s).all()
        keep = np.asarray(p.ref.len) - rng.integers(0, 6, 5)
        p.truncate(keep)
