"""The binding's short way takes the calls that its long way takes, with the same results, and leaves what is not in order to
the long way, which refuses it."""
import threading

import pytest

from paper_2406_06385_gb300 import lrqat as LQ

from gpu_util import torch

pytestmark = pytest.mark.gpu


class Calls:
    """Arguments of every call of the short way, in order; `out`: the places of what it writes."""

    def __init__(self):
        t = torch()
        t.manual_seed(0)
        LQ.lib()
        ints = lambda v, dt=t.int32: t.tensor(v, dtype=dt, device="cuda")  # noqa: E731
        bf = lambda *n: t.randn(*n, device="cuda").bfloat16()  # noqa: E731
        room = lambda n: t.empty(n, dtype=t.uint8, device="cuda")  # noqa: E731
        f32 = lambda n: t.zeros(n, device="cuda")  # noqa: E731
        hq, hk, d, P, T = 8, 2, 128, 16, 12
        rope = LQ.QKRope.of(hq, hk, d, LQ.rope_turns([10000.0 ** (-i / 64) for i in range(64)]).cuda())
        pos, g = ints(list(range(T))), [bf(d), bf(d)]
        fwd = [rope, pos, bf(T, hq, d), bf(T, hk, d), *g, bf(T, hq, d), bf(T, hk, d)]
        bwd = [rope, pos, bf(T, hq, d), bf(T, hk, d), bf(T, hq, d), bf(T, hk, d), *g, bf(T, hq, d), bf(T, hk, d), f32(d), f32(d),
               False, room(LQ.qk_rope_bwd_workspace_bytes(rope, T))]
        table, ids = t.arange(120, device="cuda").int().view(3, 40), t.arange(120, 160, device="cuda").int()
        blocks = LQ.KVBlocks.of(table, ids, P, 0)
        ws = room(LQ.kv_blocks_workspace_bytes(blocks))
        extend = [blocks, ints([600, 600, 600]), ints([1, 4, -1]), ints([40]), ints([0] * 3), ints([0]), ints([0] * 3), ints([0] * 4),
                  ints([0] * 6), ints([0] * 6, t.int64), ws]
        truncate = [blocks, ints([600, 600, 600]), ints([550, 600, 130]), ints([2]), ints([0] * 3), ints([0]), ws]
        codes = [t.randint(-127, 128, (160, hk, P, d), dtype=t.int8, device="cuda") for _ in range(2)]
        scale = [t.rand(160, hk, device="cuda") * 0.01 for _ in range(2)]
        cache = LQ.KVCache.of(*codes, *scale)
        batch = LQ.KVBatch.of(ints([600, 590, 0]), ints([0, 5, 11, 12]), table, T, 6, 640)
        n = LQ.kv_attn_sinks_workspace_bytes(cache, batch, hq, 100, 4)
        sinks = [cache, batch, bf(T, hq, d), 0.1, 100, 4, bf(T, hq, d), room(n)]
        n = LQ.kv_attn_shared_workspace_bytes(cache, batch, hq, 528)
        shared = [cache, batch, t.arange(33, device="cuda").int(), 528, bf(T, hq, d), 0.1, bf(T, hq, d), room(n)]
        self.args = dict(qk_rope_fwd=fwd, qk_rope_bwd=bwd, kv_extend=extend, kv_truncate=truncate, kv_attn_sinks=sinks,
                         kv_attn_shared=shared)
        self.out = dict(qk_rope_fwd=(6, 7), qk_rope_bwd=(8, 9, 10, 11), kv_extend=(4, 5, 6, 7, 8, 9), kv_truncate=(4, 5),
                        kv_attn_sinks=(6,), kv_attn_shared=(6,))
        self.structures = dict(fill_cache=(LQ.KVCache, [*codes, *scale]),
                               fill_batch=(LQ.KVBatch, [*batch.tensors, T, 6, 640]),
                               fill_blocks=(LQ.KVBlocks, [table, ids, P, 0]))
        self.sizes = dict(kv_attn_sinks_workspace_bytes=[cache, batch, hq, 100, 4], kv_blocks_workspace_bytes=[blocks],
                          kv_attn_shared_workspace_bytes=[cache, batch, hq, 528], qk_rope_bwd_workspace_bytes=[rope, T])


NAMES = ["qk_rope_fwd", "qk_rope_bwd", "kv_extend", "kv_truncate", "kv_attn_sinks", "kv_attn_shared"]


@pytest.fixture(scope="module")
def calls():
    return Calls()


@pytest.mark.parametrize("name", NAMES)
def test_same_results_as_the_long_way(calls, name, monkeypatch):
    t = torch()
    args, results = calls.args[name], []
    for short in (True, False):
        for i in calls.out[name]:
            args[i].zero_()
        if short:
            assert getattr(LQ._short, name)(*args) == 0
        else:
            monkeypatch.setattr(LQ, "_short", None)
            getattr(LQ, name)(*args)
        LQ.get_device_status()
        results.append([args[i].clone() for i in calls.out[name]])
    assert all(t.equal(a, b) for a, b in zip(*results)) and any(bool(a.any()) for a in results[0])


@pytest.mark.parametrize("name", ["fill_cache", "fill_batch", "fill_blocks"])
def test_structures(calls, name, monkeypatch):
    cls, args = calls.structures[name]
    a = cls()
    assert getattr(LQ._short, name)(a, *args) == 0                       # the device
    monkeypatch.setattr(LQ, "_short", None)
    assert bytes(a) == bytes(cls.of(*args))


def test_sizes(calls, monkeypatch):
    for name, args in calls.sizes.items():
        size = getattr(LQ._short, name)(*args)
        with monkeypatch.context() as m:
            m.setattr(LQ, "_short", None)
            assert size == getattr(LQ, name)(*args)


@pytest.mark.parametrize("name", ["fill_cache", "fill_batch", "fill_blocks"])
def test_bytes_are_no_structure(calls, name):
    """Nothing is written into what only has a structure's size."""
    cls, args = calls.structures[name]
    room = bytearray(bytes(cls()))
    assert getattr(LQ._short, name)(room, *args) is None and not any(room)


def _others(t, x):
    """What is not in order where the tensor x is."""
    yield x.cpu()
    yield x.to(t.float64)
    yield x.to(t.complex64)
    yield None
    yield 5
    if x.dim() == 1 and x.numel() > 1:
        yield x[:-1]
        yield x.repeat_interleave(2)[::2]
    if x.dim() > 1:
        yield x[..., :-1]
        yield x.transpose(-1, -2)
        yield x[:-1]
        yield x.unsqueeze(0)
        yield x.repeat_interleave(2, -1)[..., ::2]


# None is an argument: no gamma, no positions, no slots, no dgamma; a gradient without a gamma needs no input, a window
# that is not cut no workspace
OPTIONAL = dict(qk_rope_fwd=(1, 4, 5), qk_rope_bwd=(1, 4, 5, 6, 7, 10, 11, 13), kv_extend=(9,), kv_attn_sinks=(7,))


@pytest.mark.parametrize("name", NAMES)
def test_what_is_not_in_order(calls, name):
    """Refused before anything runs: the short way says nothing or passes on the library's refusal, the long way raises."""
    t = torch()
    good = calls.args[name]
    for i, x in enumerate(good):
        if not isinstance(x, t.Tensor):
            continue
        room = x.dtype is t.uint8
        for bad in _others(t, x):
            if bad is None and i in OPTIONAL.get(name, ()) or room and isinstance(bad, t.Tensor) and (bad.is_cuda or bad.dim() > 1):
                continue
            args = good[:i] + [bad] + good[i + 1:]
            if name == "kv_extend" and i == 8 and isinstance(bad, t.Tensor) and bad.dtype is x.dtype and bad.is_cuda and bad.is_contiguous():
                continue                                                  # fewer rows are a call of their own
            got = getattr(LQ._short, name)(*args)
            assert got is None or got < 0, (name, i, bad)
            with pytest.raises((LQ.LrqatError, AttributeError, TypeError)):
                getattr(LQ, name)(*args)
    LQ.get_device_status()
    assert getattr(LQ._short, name)(*good[:-1]) is None and getattr(LQ._short, name)(*good, None) is None
    assert getattr(LQ._short, name)(object(), *good[1:]) is None and getattr(LQ._short, name)(b"x", *good[1:]) is None
    for i, x in enumerate(good):
        if isinstance(x, (int, float)) and not isinstance(x, bool):
            for bad in ("x", None, 1 << 40, 1 << 70):
                got = getattr(LQ._short, name)(*good[:i], bad, *good[i + 1:])
                assert got is None


@pytest.mark.parametrize("name", ["qk_rope_fwd", "qk_rope_bwd"])
def test_turns_of_another_device(calls, name, monkeypatch):
    """As the rotation says where they lie: the addresses are this device's."""
    args = calls.args[name]
    monkeypatch.setattr(args[0], "device", 1)
    assert getattr(LQ._short, name)(*args) is None
    with pytest.raises(LQ.LrqatError) as e:
        getattr(LQ, name)(*args)
    assert e.value.status == -1
    for other in ("x", 1 << 70):
        monkeypatch.setattr(args[0], "device", other)
        assert getattr(LQ._short, name)(*args) is None
    for fine in (0, None):
        monkeypatch.setattr(args[0], "device", fine)
        assert getattr(LQ._short, name)(*args) == 0
    LQ.get_device_status()


@pytest.mark.parametrize("name", [n for n in NAMES if n != "qk_rope_fwd"])
def test_workspaces_that_are_not_there(calls, name):
    """One element, expanded: its bytes are counted, and would be written behind it."""
    good = calls.args[name]
    (i,) = [i for i, x in enumerate(good) if isinstance(x, torch().Tensor) and x.dtype is torch().uint8]
    room = torch().empty(1 << 21, dtype=torch().uint8, device="cuda")         # a window that is not cut needs none
    for bad in (room[:1].expand(1 << 20), room[::2]):
        args = good[:i] + [bad] + good[i + 1:]
        assert getattr(LQ._short, name)(*args) is None
        with pytest.raises(LQ.LrqatError) as e:
            getattr(LQ, name)(*args)
        assert e.value.status == -1


def test_structures_that_are_not_in_order(calls):
    t = torch()
    for name, (cls, good) in calls.structures.items():
        for i, x in enumerate(good):
            if not isinstance(x, t.Tensor):
                continue
            for bad in _others(t, x):
                if name == "fill_blocks" and isinstance(bad, t.Tensor) and bad.is_cuda and bad.dtype is x.dtype and bad.is_contiguous() \
                        and bad.dim() == x.dim():
                    continue                                              # another list of blocks
                if name == "fill_batch" and i == 2 and isinstance(bad, t.Tensor) and bad.shape[:1] == x.shape[:1] and bad.is_contiguous() \
                        and bad.dtype is x.dtype and bad.dim() == 2 and bad.is_cuda:
                    continue                                              # a narrower table
                args = good[:i] + [bad] + good[i + 1:]
                a = cls()
                before = bytes(a)
                assert getattr(LQ._short, name)(a, *args) is None and bytes(a) == before, (name, i, bad)


def test_two_threads(calls):
    """Calls of two threads, each on a stream of its own with outputs and workspace of its own."""
    t = torch()
    cache, batch, table, prefix, Q, scale, _, ws = calls.args["kv_attn_shared"]
    want = t.empty_like(Q)
    LQ.kv_attn_shared(cache, batch, table, prefix, Q, scale, want, ws)
    t.cuda.synchronize()
    bad = []

    def work():
        try:
            with t.cuda.stream(t.cuda.Stream()):
                for _ in range(50):
                    out, room = t.empty_like(Q), t.empty_like(ws)
                    LQ.kv_attn_shared(cache, batch, table, prefix, Q, scale, out, room)
                    if not t.equal(out, want):
                        bad.append("another result")
        except Exception as e:  # noqa: BLE001
            bad.append(e)

    threads = [threading.Thread(target=work) for _ in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not bad
