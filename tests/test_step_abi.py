"""The block table and head rotation entry points reject bad arguments on the host before any CUDA work."""
import ctypes
import math
import os
import sys
import types

import pytest

import paper_2406_06385_gb300.build as B
from paper_2406_06385_gb300 import lrqat as LQ
from paper_2406_06385_gb300.build import build

OK = 16   # a 16-byte aligned address that is never followed


@pytest.fixture(scope="module")
def lib():
    build()
    return LQ.lib()


def _rope(**kw):
    return LQ.QKRope(**dict(dict(n_heads=4, n_kv_heads=2, head_dim=128, rot_dim=128, neighbours=0, eps=1e-6, turns=OK), **kw))


def _fwd(lib, rope, T=4, pos=OK, Q=OK, ldq=512, K=OK, ldk=256, gq=OK, gk=OK, Qo=OK, ldqo=512, Ko=OK, ldko=256):
    return lib.lrqat_qk_rope_fwd(ctypes.byref(rope), T, pos, Q, ldq, K, ldk, gq, gk, Qo, ldqo, Ko, ldko, None)


def _bwd(lib, rope, T=4, pos=OK, dQo=OK, lddqo=512, dKo=OK, lddko=256, Q=OK, ldq=512, K=OK, ldk=256, gq=OK, gk=OK, dQ=OK,
         lddq=512, dK=OK, lddk=256, dgq=OK, dgk=OK, ws=OK, size=1 << 30):
    return lib.lrqat_qk_rope_bwd(ctypes.byref(rope), T, pos, dQo, lddqo, dKo, lddko, Q, ldq, K, ldk, gq, gk, dQ, lddq, dK,
                                 lddk, dgq, dgk, 0, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n_heads=-1), -1), (dict(n_heads=0, n_kv_heads=0), -1), (dict(n_kv_heads=16385), -2), (dict(head_dim=0), -1),
    (dict(head_dim=72, rot_dim=0), -2), (dict(head_dim=272), -2), (dict(rot_dim=136), -1), (dict(rot_dim=-16), -1),
    (dict(rot_dim=8), -2), (dict(neighbours=2), -1), (dict(eps=-1.0), -1), (dict(eps=float("inf")), -1),
    (dict(eps=float("nan")), -1), (dict(turns=None), -1), (dict(turns=20), -3)])
def test_rope_settings(lib, kw, status):
    assert _fwd(lib, _rope(**kw)) == status and LQ.last_error()
    assert _bwd(lib, _rope(**kw)) == status
    assert lib.lrqat_qk_rope_bwd_workspace_bytes(ctypes.byref(_rope(**kw)), 4) == 0


def test_rope_arrays(lib):
    r = _rope()
    for call in (_fwd, _bwd):
        assert call(lib, r, T=0) == -1 and call(lib, r, T=1 << 31) == -2 and call(lib, r, pos=18) == -3
        for name in ("Q", "K"):
            assert call(lib, r, **{name: None}) == -1 and call(lib, r, **{name: 24}) == -3
        for name, row in (("ldq", 512), ("ldk", 256)):
            assert call(lib, r, **{name: row - 8}) == -1 and call(lib, r, **{name: row + 4}) == -3
        for name in ("gq", "gk"):
            assert call(lib, r, **{name: 24}) == -3
    for name in ("Qo", "Ko"):
        assert _fwd(lib, r, **{name: None}) == -1 and _fwd(lib, r, **{name: 24}) == -3
    for name in ("dQo", "dKo", "dQ", "dK"):
        assert _bwd(lib, r, **{name: None}) == -1 and _bwd(lib, r, **{name: 24}) == -3
    for name, row in (("lddqo", 512), ("lddko", 256), ("lddq", 512), ("lddk", 256)):
        assert _bwd(lib, r, **{name: row - 8}) == -1 and _bwd(lib, r, **{name: row + 4}) == -3
    need = lib.lrqat_qk_rope_bwd_workspace_bytes(ctypes.byref(r), 4)
    assert need > 0 and _bwd(lib, r, ws=None) == -4 and _bwd(lib, r, size=need - 1) == -4 and _bwd(lib, r, ws=24) == -3
    assert _bwd(lib, r, dgq=24) == -3 and _bwd(lib, r, gq=None) == -1           # dgamma without gamma
    assert _bwd(lib, _rope(n_kv_heads=0), dgk=OK) == -1


def test_outputs_that_overlap_other_arrays(lib):
    """Parts of one array, 4 heads for queries, 2 for keys and 2 for values, are apart; so are an output and its own input,
    where rows are as far apart.  Addresses are never followed: the calls that pass end at the device."""
    try:
        import torch
        if torch.cuda.is_available():
            pytest.skip("calls that pass would run")
    except ImportError:
        pass
    r, at = _rope(), lambda array, element=0: 16 + (array << 20) + 2 * element
    part = dict(ldq=1024, ldk=1024, ldqo=1024, ldko=1024)
    fwd = lambda Q, K, Qo, Ko, **kw: _fwd(lib, r, Q=Q, K=K, Qo=Qo, Ko=Ko, **dict(part, **kw))  # noqa: E731
    passes = -5                                                    # no device
    q, k = at(1), at(1, 512)
    assert fwd(q, k, q, k) == passes and fwd(q, k, at(2), at(2, 512)) == passes
    assert fwd(q, k, at(2), at(3), ldqo=512, ldko=256) == passes
    assert fwd(q, k, at(2), at(2, 504)) == -1 and "overlap" in LQ.last_error()     # a head's end over the keys
    assert fwd(q, k, at(1, 8), at(2)) == -1 and fwd(q, k, at(2), q) == -1 and fwd(q, k, k, at(2)) == -1
    assert fwd(q, k, q, at(2), ldqo=512) == -1                     # in place, rows at other distances
    assert fwd(q, k, q, at(2), ldqo=512, T=1) == passes
    assert fwd(q, k, at(1, 4 * 1024), at(2)) == passes and fwd(q, k, at(1, 3 * 1024), at(2)) == -1
    assert fwd(at(1, 768), at(2), at(1), at(3)) == -1 and fwd(at(1, 512), at(2), at(1), at(3)) == passes
    bwd = lambda dQo, dKo, Q, K, dQ, dK, **kw: _bwd(lib, r, dQo=dQo, dKo=dKo, Q=Q, K=K, dQ=dQ, dK=dK, dgk=64, **kw)  # noqa: E731
    a = [at(i) for i in range(1, 7)]
    assert bwd(*a) == passes and bwd(*a[:4], a[0], a[1]) == passes and bwd(*a[:4], a[2], a[3]) == passes
    for dq, dk in ((a[1], a[5]), (a[3], a[5]), (a[4], a[0]), (a[4], a[2]), (a[4], a[4])):
        assert bwd(*a[:4], dq, dk) == -1
    assert bwd(*a[:4], a[0], a[5], lddq=1024) == -1
    assert _bwd(lib, r, dQo=a[0], dKo=a[1], Q=a[2], K=a[3], dQ=a[4], dK=a[5]) == -1        # one dgamma for both
    # the inputs of heads without a norm are not read
    assert bwd(*a[:4], a[4], a[2], gq=None, dgq=None) == passes


def test_outputs_that_overlap_flat_arrays(lib):
    """Positions, turns, gammas, and behind the gradient dgamma and the workspace: apart from every row of an output, but they
    may lie between rows.  Addresses are never followed: the calls that pass end at the device."""
    try:
        import torch
        if torch.cuda.is_available():
            pytest.skip("calls that pass would run")
    except ImportError:
        pass
    T, passes = 4, -5                                              # no device
    at = lambda array, byte=0: 16 + (array << 20) + byte           # noqa: E731
    flat = dict(pos=at(10), gq=at(11), gk=at(12))
    rows = dict(Q=at(1), K=at(2), Qo=at(3), Ko=at(4), ldqo=1024, ldko=1024)

    def fwd(turns=at(13), **kw):
        return _fwd(lib, _rope(turns=turns), T=T, **{**rows, **flat, **kw})

    bwd_rows = dict(dQo=at(1), dKo=at(2), Q=at(5), K=at(6), dQ=at(3), dK=at(4), lddq=1024, lddk=1024)
    sums = dict(dgq=at(14), dgk=at(15), ws=at(16))

    def bwd(turns=at(13), **kw):
        return _bwd(lib, _rope(turns=turns), T=T, **{**bwd_rows, **flat, **sums, **kw})

    assert fwd() == passes and bwd() == passes
    # rows of 1024 (512) bytes, 2048 bytes apart: places at a row's start, at its end, between rows, in the last row, behind it
    for array, width in ((3, 1024), (4, 512)):
        for call, names in ((fwd, ("pos", "turns", "gq", "gk")), (bwd, ("pos", "turns", "gq", "gk", "dgq", "dgk", "ws"))):
            for name in names:
                size = dict(pos=4 * T, turns=512, gq=256, gk=256, dgq=512, dgk=512, ws=1 << 18)[name]
                place = lambda byte: call(**{name: at(array, byte)})  # noqa: E731
                for byte in (0, width - 16, 2048, 3 * 2048 + width - 16, -16 if size > 16 else 0):
                    assert place(byte) == -1 and "overlap" in LQ.last_error(), (array, name, byte)
                assert place(3 * 2048 + width) == passes
                if name != "ws":
                    assert place(width) == passes and place(2048 + width) == passes and place(-size) == passes
    # what is written lies apart from the inputs' rows as well; what is read may lie anywhere among them
    for array, width in ((1, 1024), (2, 512), (5, 1024), (6, 512)):
        for name in ("dgq", "dgk", "ws"):
            for byte in (0, 3 * width, 4 * width - 16):
                assert bwd(**{name: at(array, byte)}) == -1
            assert bwd(**{name: at(array, 4 * width)}) == passes
        assert bwd(pos=at(array), turns=at(array), gq=at(array), gk=at(array)) == passes
    assert fwd(gq=at(1), gk=at(1), pos=at(2)) == passes
    # without sums there is no workspace, and inputs of heads without a norm are not read
    assert bwd(dgq=None, dgk=None, ws=at(3)) == passes and bwd(gq=None, dgq=None, Q=at(14), dgk=at(14, 64)) == passes


def test_turns_of_frequencies(lib):
    """Exact to half a unit of 2^-64 turns (pi to 87 digits), wrapped around, for either sign."""
    from fractions import Fraction
    turn = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803")
    freq = [1.0, 0.5, 10000.0 ** (-2 / 128), 500000.0 ** -0.9, 1e-300, 5e-324, 0.0, -0.3, 2.0 ** 20, -2.0 ** 20, 2 * math.pi, 1e-15]
    for f, t in zip(freq, LQ.rope_turns(freq).tolist()):
        assert abs(Fraction(t) - (x := Fraction(f) / turn * 2 ** 64) + 2 ** 64 * round((x - t) / 2 ** 64)) <= Fraction(51, 100)
    for bad in (float("nan"), float("inf"), 2.0 ** 20 + 1, -1e9):
        with pytest.raises(LQ.LrqatError) as e:
            LQ.rope_turns([1.0, bad])
        assert e.value.status == -1
    assert lib.lrqat_rope_turns(None, 0, None) == 0 and lib.lrqat_rope_turns(None, 1, None) == -1
    assert lib.lrqat_rope_turns(None, -1, None) == -1


def _blocks(**kw):
    return LQ.KVBlocks(**dict(dict(n_seqs=3, max_blocks=4, block=16, pinned=0, capacity=64, block_table=OK, free_ids=OK), **kw))


def _extend(lib, b, n=OK, add=32, count=OK, rows=5, n_out=OK, count_out=OK, seen=48, start=64, pos=80, slot=96, ws=OK, size=1 << 20):
    return lib.lrqat_kv_extend(ctypes.byref(b), n, add, count, rows, n_out, count_out, seen, start, pos, slot, ws, size, None)


def _truncate(lib, b, n=OK, keep=OK, count=OK, n_out=OK, count_out=OK, ws=OK, size=1 << 20):
    return lib.lrqat_kv_truncate(ctypes.byref(b), n, keep, count, n_out, count_out, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n_seqs=0), -1), (dict(n_seqs=65536), -2), (dict(max_blocks=0), -1), (dict(max_blocks=1 << 27), -2),
    (dict(block=8), -2), (dict(block=24), -2), (dict(pinned=-1), -1), (dict(pinned=5), -1), (dict(capacity=0), -1),
    (dict(capacity=(1 << 31) - 1), -2), (dict(block_table=None), -1), (dict(free_ids=None), -1), (dict(free_ids=18), -3)])
def test_block_settings(lib, kw, status):
    assert _extend(lib, _blocks(**kw)) == status and LQ.last_error()
    assert _truncate(lib, _blocks(**kw)) == status
    assert lib.lrqat_kv_blocks_workspace_bytes(ctypes.byref(_blocks(**kw))) == 0


def test_block_arrays(lib):
    b = _blocks()
    for call, change in ((_extend, "add"), (_truncate, "keep")):
        for name in ("n", change, "count", "n_out", "count_out"):
            assert call(lib, b, **{name: None}) == -1 and call(lib, b, **{name: 18}) == -3
        need = lib.lrqat_kv_blocks_workspace_bytes(ctypes.byref(b))
        assert need > 0 and call(lib, b, ws=None) == -4 and call(lib, b, size=need - 1) == -4 and call(lib, b, ws=24) == -3
    for name in ("seen", "start", "pos"):
        assert _extend(lib, b, **{name: None}) == -1 and _extend(lib, b, **{name: 18}) == -3
    assert _extend(lib, b, slot=20) == -3 and _extend(lib, b, rows=-1) == -1 and _extend(lib, b, rows=(1 << 31) - 1) == -2
    assert _extend(lib, b, seen=OK) == -1                     # the batch's lengths over the sequences'


def _stand_in(torch, shape, dtype, device="cuda:0"):
    """What the binding asks of a tensor, with an address that is never followed."""
    t = torch.zeros(shape, dtype=dtype)
    return types.SimpleNamespace(shape=t.shape, dtype=dtype, stride=t.stride, numel=t.numel, element_size=t.element_size,
                                 dim=t.dim, is_contiguous=t.is_contiguous, is_cuda=device != "cpu",
                                 device=torch.device(device), data_ptr=lambda: OK,
                                 get_device=lambda: -1 if device == "cpu" else int(device[5:]))


@pytest.fixture
def recorded(monkeypatch):
    """The binding with a library that only notes its calls; device 0 is the current one."""
    torch = pytest.importorskip("torch")
    calls = []
    record = lambda name: lambda *a: calls.append((name, a)) or 0  # noqa: E731
    monkeypatch.setattr(LQ, "lib", lambda: types.SimpleNamespace(**{n: record(n) for n in (
        "lrqat_qk_rope_fwd", "lrqat_qk_rope_bwd", "lrqat_kv_extend", "lrqat_kv_truncate")}))
    monkeypatch.setattr(LQ, "_current_device", lambda: 0)
    return torch, calls, lambda shape, dtype, device="cuda:0": _stand_in(torch, shape, dtype, device)


def test_the_short_way_leaves_what_it_does_not_know(lib):
    """Without CUDA tensors it says nothing and writes nothing, whatever it is given."""
    torch = pytest.importorskip("torch")
    LQ.lib()
    if LQ._short is None:
        pytest.skip("not built for this torch")
    codes, scale, ints = torch.zeros(2, 1, 16, 64, dtype=torch.int8), torch.zeros(2, 1), torch.zeros(2, 1, dtype=torch.int32)
    cache, batch, blocks = LQ.KVCache(), LQ.KVBatch(), LQ.KVBlocks()
    for of, args in ((LQ._short.fill_cache, (cache, codes, codes, scale, scale)),
                     (LQ._short.fill_batch, (batch, ints[:, 0], torch.zeros(3, dtype=torch.int32), ints, 2, 1, 16)),
                     (LQ._short.fill_blocks, (blocks, ints, ints[:, 0], 16, 0))):
        assert of(*args) is None and not any(bytes(args[0]))
        for i in range(len(args)):
            assert of(*args[:i], None, *args[i + 1:]) is None and of(*args[:i], object(), *args[i + 1:]) is None
        assert of() is None and of(*args, 1) is None
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    assert LQ._short.kv_attn_sinks(cache, batch, q, 0.1, 0, 0, q, None) is None
    assert LQ._short.kv_attn_shared(cache, batch, None, 0, q, 0.1, q, None) is None
    assert LQ._short.qk_rope_fwd(_rope(head_dim=64, rot_dim=64), None, q, q[:, :2], None, None, q, q[:, :2]) is None
    assert LQ._short.kv_extend(blocks, *[ints] * 8, None, None) is None and LQ._short.kv_truncate(blocks, *[ints] * 5, None) is None
    # sizes need no tensors, and are the library's
    assert LQ._short.kv_blocks_workspace_bytes(_blocks()) == lib.lrqat_kv_blocks_workspace_bytes(ctypes.byref(_blocks())) > 0
    assert LQ._short.qk_rope_bwd_workspace_bytes(_rope(), 4) == lib.lrqat_qk_rope_bwd_workspace_bytes(ctypes.byref(_rope()), 4) > 0
    assert LQ._short.kv_blocks_workspace_bytes(_rope()) is None and LQ._short.qk_rope_bwd_workspace_bytes(_rope(), 1.5) is None


def test_a_short_way_that_does_not_load_is_done_without(lib, monkeypatch, tmp_path):
    """As one that was built for a torch with CUDA does not load with the same version of torch without."""
    torch = pytest.importorskip("torch")
    name = f"lrqat_binding-{torch.__version__.split('+')[0]}-{sys.implementation.cache_tag}.so"
    (tmp_path / name).write_bytes(b"\x7fELF")
    monkeypatch.setattr(LQ, "LIB_PATH", str(tmp_path / "liblrqat.so"))
    assert LQ._load_short() is None
    monkeypatch.setattr(LQ, "_short", LQ._short)
    monkeypatch.setattr(LQ, "_short_tried", False)
    assert LQ.lib() is lib and LQ._short is None


@pytest.mark.parametrize("command", [["false"], ["no-such-compiler"]])
def test_a_short_way_that_does_not_compile_is_done_without(lib, monkeypatch, tmp_path, capsys, command):
    """The library is there all the same, and no short way of older sources beside it."""
    old = tmp_path / "lrqat_binding.so"
    old.write_bytes(b"")
    os.utime(old, (1, 1))
    monkeypatch.setattr(B, "binding_path", lambda: str(old))
    monkeypatch.setattr(B, "binding_command", lambda target: command)
    assert B.build() == B.LIB_PATH and os.path.exists(B.LIB_PATH)
    assert not old.exists() and "does without" in capsys.readouterr().err


def test_the_short_way_takes_the_bindings_structures_only(lib):
    """Bytes of a structure's size are not one: the long way takes none either."""
    pytest.importorskip("torch")
    LQ.lib()
    if LQ._short is None:
        pytest.skip("not built for this torch")

    class MyBlocks(LQ.KVBlocks):
        pass

    class Twin(ctypes.Structure):
        _fields_ = LQ.KVBlocks._fields_

    size, blocks, rope = LQ._short.kv_blocks_workspace_bytes, _blocks(), _rope()
    for other in (bytes(blocks), bytearray(blocks), memoryview(bytes(blocks)), Twin.from_buffer_copy(blocks), (ctypes.c_char * 40)()):
        assert size(other) is None
    assert size(MyBlocks.from_buffer_copy(blocks)) == size(blocks) > 0
    assert LQ._short.qk_rope_bwd_workspace_bytes(bytes(rope), 4) is None
    sinks, shared = LQ._short.kv_attn_sinks_workspace_bytes, LQ._short.kv_attn_shared_workspace_bytes
    assert sinks(_cache(), _batch(), 4, 0, 0) is not None and shared(_cache(), _batch(), 4, 16) is not None
    for c, b in ((bytes(_cache()), _batch()), (_cache(), bytes(_batch())), (_batch(), _batch()), (_cache(), _cache())):
        assert sinks(c, b, 4, 0, 0) is None and shared(c, b, 4, 16) is None
    for bad in ((), (int,), (int, int, int, 5)):
        with pytest.raises(TypeError):
            LQ._short.structures(*bad)
    assert size(blocks) > 0


def test_binding_checks_rope_arrays(recorded):
    torch, calls, fake = recorded
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    turns = fake((64,), torch.int64)
    rope = LQ.QKRope.of(4, 2, 128, turns)
    assert rope.rot_dim == 128 and LQ.QKRope.of(4, 2, 128, None).rot_dim == 0
    for bad in (fake((64,), torch.float64), fake((64, 2), torch.int64), fake((64,), torch.int64, "cpu")):
        with pytest.raises(LQ.LrqatError):
            LQ.QKRope.of(4, 2, 128, bad)
    good = dict(pos=fake((6,), i32), Q=fake((6, 4, 128), bf), K=fake((6, 2, 128), bf), gq=fake((128,), bf),
                gk=fake((128,), torch.int16), Qo=fake((6, 4, 128), bf), Ko=fake((6, 2, 128), torch.int16),
                dgq=fake((128,), f32), dgk=fake((128,), f32), ws=fake((4096,), torch.uint8))

    def fwd(**kw):
        a = {**good, **kw}
        LQ.qk_rope_fwd(rope, a["pos"], a["Q"], a["K"], a["gq"], a["gk"], a["Qo"], a["Ko"], stream=0)

    def bwd(**kw):
        a = {**good, **kw}
        LQ.qk_rope_bwd(rope, a["pos"], a["Qo"], a["Ko"], a["Q"], a["K"], a["gq"], a["gk"], a["Qo"], a["Ko"], a["dgq"],
                       a["dgk"], False, a["ws"], stream=0)

    for call in (fwd, bwd):
        call()
        call(pos=None)
        call(gq=None, dgq=None, gk=fake((200,), bf))
        for name, shape, dtype in (("Q", (6, 4, 128), bf), ("K", (6, 2, 128), bf), ("Qo", (6, 4, 128), bf), ("Ko", (6, 2, 128), bf)):
            for bad in (fake(shape, f32), fake(shape, dtype, "cpu"), fake(shape, dtype, "cuda:1"), fake((5,) + shape[1:], dtype),
                        fake((6, 3, 128), dtype), None):
                with pytest.raises(LQ.LrqatError):
                    call(**{name: bad})
        for bad in (fake((5,), i32), fake((6,), torch.int64), fake((6,), i32, "cpu"), fake((6,), i32, "cuda:1")):
            with pytest.raises(LQ.LrqatError):
                call(pos=bad)
        for bad in (fake((127,), bf), fake((128,), f32), fake((128,), bf, "cpu")):
            with pytest.raises(LQ.LrqatError):
                call(gk=bad)
        for device in ("cuda:1",):                            # all on another device than the current one
            with pytest.raises(LQ.LrqatError):
                call(**{n: fake(t.shape, t.dtype, device) for n, t in good.items()})
    for kw in (dict(dgq=fake((127,), f32)), dict(dgk=fake((128,), bf)), dict(ws=fake((64,), torch.uint8, "cpu"))):
        with pytest.raises(LQ.LrqatError):
            bwd(**kw)
    assert len(calls) == 6


def test_binding_checks_the_device_of_the_turns(recorded):
    """Angles of another device than the call's arrays would be followed as an address of this one."""
    torch, calls, fake = recorded
    q, g, dg, ws = fake((6, 1, 16), torch.bfloat16), fake((16,), torch.bfloat16), fake((16,), torch.float32), fake((4096,), torch.uint8)

    def run(rope):
        yield lambda: LQ.qk_rope_fwd(rope, None, q, None, g, None, q, None, stream=0)
        yield lambda: LQ.qk_rope_bwd(rope, None, q, None, q, None, g, None, q, None, dg, None, False, ws, stream=0)

    here, elsewhere = (LQ.QKRope.of(1, 0, 16, fake((8,), torch.int64, device)) for device in ("cuda:0", "cuda:1"))
    assert (here.device, elsewhere.device, LQ.QKRope.of(1, 0, 16, None).device) == (0, 1, None)
    by_hand = LQ.QKRope(1, 0, 16, 16, 0, 0.0, OK)
    for rope in (here, LQ.QKRope.of(1, 0, 16, None), by_hand):
        for call in run(rope):
            call()
    assert len(calls) == 6
    for call in run(elsewhere):
        with pytest.raises(LQ.LrqatError) as e:
            call()
        assert e.value.status == -1
    assert len(calls) == 6


def test_binding_checks_block_arrays(recorded):
    torch, calls, fake = recorded
    i32 = torch.int32
    table, free = fake((3, 4), i32), fake((64,), i32)
    blocks = LQ.KVBlocks.of(table, free, 16, 1)
    assert (blocks.n_seqs, blocks.max_blocks, blocks.capacity, blocks.pinned) == (3, 4, 64, 1)
    for bad in ((fake((3, 4), torch.int64), free), (table, fake((64,), torch.int64)), (fake((12,), i32), free),
                (table, fake((8, 8), i32)), (fake((3, 4), i32, "cpu"), fake((64,), i32, "cpu")), (table, fake((64,), i32, "cuda:1"))):
        with pytest.raises(LQ.LrqatError):
            LQ.KVBlocks.of(*bad, 16)
    n = lambda k, dtype=i32, device="cuda:0": fake((k,), dtype, device)  # noqa: E731
    names = ["lens", "add", "free_count", "lens_out", "free_out", "batch_lens", "row_start", "pos", "slot", "workspace"]
    good = dict(zip(names, [n(3), n(3), n(1), n(3), n(1), n(3), n(4), n(7), n(7, torch.int64), n(64, torch.uint8)]))
    LQ.kv_extend(blocks, **good, stream=0)
    LQ.kv_extend(blocks, **{**good, "slot": None}, stream=0)
    assert calls[0][1][4] == 7 and calls[1][1][10] is None
    keep = [good[k] for k in ("lens", "add", "free_count", "lens_out", "free_out", "workspace")]
    LQ.kv_truncate(blocks, *keep, stream=0)
    for name, size in zip(names[:9], (3, 3, 1, 3, 1, 3, 4, 7, 7)):
        dtype = torch.int64 if name == "slot" else i32
        bad = [n(size, torch.int16), n(size, dtype, "cpu"), n(size, dtype, "cuda:1")] + ([n(size - 1, dtype)] if name != "pos" else [])
        for t in bad + ([None] if name != "slot" else []):
            with pytest.raises(LQ.LrqatError):
                LQ.kv_extend(blocks, **{**good, name: t}, stream=0)
            if names.index(name) < 5:
                with pytest.raises(LQ.LrqatError):
                    LQ.kv_truncate(blocks, *[t if i == names.index(name) else v for i, v in enumerate(keep)], stream=0)
    with pytest.raises(LQ.LrqatError):
        LQ.kv_extend(blocks, **{**good, "workspace": n(64, torch.uint8, "cpu")}, stream=0)
    assert len(calls) == 3


def test_binding_refuses_another_device_than_the_current_one(recorded, monkeypatch):
    torch, calls, fake = recorded
    monkeypatch.setattr(LQ, "_current_device", lambda: 1)
    i32 = torch.int32
    blocks = LQ.KVBlocks.of(fake((3, 4), i32), fake((64,), i32), 16)
    n = lambda k: fake((k,), i32)  # noqa: E731
    with pytest.raises(LQ.LrqatError):
        LQ.kv_truncate(blocks, n(3), n(3), n(1), n(3), n(1), fake((64,), torch.uint8), stream=0)
    q = fake((2, 1, 16), torch.bfloat16)
    with pytest.raises(LQ.LrqatError):
        LQ.qk_rope_fwd(LQ.QKRope.of(1, 0, 16, None), None, q, None, None, None, q, None, stream=0)
    assert not calls


def _cache(**kw):
    return LQ.KVCache(**dict(dict(n_blocks=8, n_kv_heads=2, head_dim=128, block=16, k_codes=OK, v_codes=OK,
                                  k_scale=OK, v_scale=OK), **kw))


def _batch(**kw):
    return LQ.KVBatch(**dict(dict(n_seqs=2, max_blocks=4, len=OK, row_start=OK, block_table=OK, rows=6, max_rows=3,
                                  max_len=64), **kw))


def _sinks(lib, c=None, b=None, heads=4, scale=1.0, window=8, sinks=4, x=OK, ld=512, o=OK, ldo=512, ws=OK, size=1 << 30):
    return lib.lrqat_kv_attn_sinks(ctypes.byref(c or _cache()), ctypes.byref(b or _batch()), heads, scale, window, sinks, x, ld,
                                   o, ldo, ws, size, None)


def _shared(lib, c=None, b=None, table=OK, prefix=32, heads=4, scale=1.0, x=OK, ld=512, o=OK, ldo=512, ws=OK, size=1 << 30):
    return lib.lrqat_kv_attn_shared(ctypes.byref(c or _cache()), ctypes.byref(b or _batch()), table, prefix, heads, scale, x,
                                    ld, o, ldo, ws, size, None)


def test_attention_calls(lib):
    for call in (_sinks, _shared):
        assert call(lib, heads=0) == -1 and call(lib, heads=3) == -1
        assert call(lib, scale=float("inf")) == -1 and call(lib, scale=float("nan")) == -1
        assert call(lib, x=None) == -1 and call(lib, x=24) == -3 and call(lib, ld=504) == -1 and call(lib, ld=513) == -3
        assert call(lib, o=None) == -1 and call(lib, o=24) == -3 and call(lib, ldo=504) == -1 and call(lib, ldo=513) == -3
        assert call(lib, b=_batch(rows=0)) == 0
        for c, status in ((_cache(head_dim=96), -2), (_cache(block=8), -2), (_cache(k_codes=None), -1)):
            assert call(lib, c=c) == status
        for b, status in ((_batch(n_seqs=0), -1), (_batch(max_len=65), -1), (_batch(len=None), -1), (_batch(rows=1 << 31), -2)):
            assert call(lib, b=b) == status
    assert _sinks(lib, window=-1) == -1 and _sinks(lib, sinks=-1) == -1
    assert _shared(lib, prefix=-16) == -1 and _shared(lib, prefix=24) == -1 and _shared(lib, prefix=80) == -1
    assert _shared(lib, table=None) == -1 and _shared(lib, table=18) == -3
    long = _batch(max_blocks=4096, max_len=65536)
    c, b = ctypes.byref(_cache()), ctypes.byref(long)
    need = lib.lrqat_kv_attn_sinks_workspace_bytes(c, b, 4, 9000, 4)
    assert need > 0
    assert _sinks(lib, b=long, window=9000, ws=None, size=need) == -4 and _sinks(lib, b=long, window=9000, size=need - 1) == -4
    assert _sinks(lib, b=long, window=9000, ws=24, size=need) == -3
    need = lib.lrqat_kv_attn_shared_workspace_bytes(c, b, 4, 16000)
    assert need > 0
    assert _shared(lib, b=long, prefix=16000, ws=None, size=need) == -4
    assert _shared(lib, b=long, prefix=16000, size=need - 1) == -4 and _shared(lib, b=long, prefix=16000, ws=24, size=need) == -3
    assert lib.lrqat_kv_attn_sinks_workspace_bytes(c, b, 4, 9000, -1) == 0
    assert lib.lrqat_kv_attn_shared_workspace_bytes(c, b, 4, 16001) == 0
    # without sinks, and without a prefix, the plain call's workspace
    for window in (0, 9000):
        plain = lib.lrqat_kv_attn_workspace_bytes(c, b, 4, window)
        assert plain > 0 and plain == lib.lrqat_kv_attn_sinks_workspace_bytes(c, b, 4, window, 0)
    assert lib.lrqat_kv_attn_workspace_bytes(c, b, 4, 0) == lib.lrqat_kv_attn_shared_workspace_bytes(c, b, 4, 0)


def test_binding_checks_attention_arrays(recorded, monkeypatch):
    torch, _, fake = recorded
    calls = []
    record = lambda *a: calls.append(a) or 0  # noqa: E731
    monkeypatch.setattr(LQ, "lib", lambda: types.SimpleNamespace(lrqat_kv_attn_sinks=record, lrqat_kv_attn_shared=record))
    i32, bf = torch.int32, torch.bfloat16
    codes, scale = fake((8, 2, 16, 128), torch.int8), fake((8, 2), torch.float32)
    cache = LQ.KVCache.of(codes, codes, scale, scale)
    batch = LQ.KVBatch.of(fake((2,), i32), fake((3,), i32), fake((2, 4), i32), 6, 3, 64)
    ws, q, table = fake((64,), torch.uint8), fake((6, 4, 128), bf), fake((2,), i32)
    sinks = lambda q=q, o=q, ws=ws: LQ.kv_attn_sinks(cache, batch, q, 1.0, 8, 4, o, ws, stream=0)  # noqa: E731
    shared = lambda q=q, o=q, ws=ws, table=table: LQ.kv_attn_shared(cache, batch, table, 32, q, 1.0, o, ws, stream=0)  # noqa: E731
    for call in (sinks, shared):
        call()
        call(ws=None)
        for bad in (fake((5, 4, 128), bf), fake((6, 4, 64), bf), fake((6, 4, 128), torch.float32), fake((6, 4, 128), bf, "cpu"),
                    fake((6, 4, 128), bf, "cuda:1"), fake((6, 512), bf)):
            for kw in (dict(q=bad), dict(o=bad)):
                with pytest.raises(LQ.LrqatError) as e:
                    call(**kw)
                assert e.value.status == -1
        with pytest.raises(LQ.LrqatError):
            call(ws=fake((64,), torch.uint8, "cpu"))
        monkeypatch.setattr(LQ, "_current_device", lambda: 1)
        with pytest.raises(LQ.LrqatError):
            call()
        monkeypatch.setattr(LQ, "_current_device", lambda: 0)
    for bad in (None, fake((1,), i32), fake((2,), torch.int64), fake((2,), i32, "cpu"), fake((2,), i32, "cuda:1")):
        with pytest.raises(LQ.LrqatError):
            shared(table=bad)
    LQ.kv_attn_shared(cache, batch, None, 0, q, 1.0, q, ws, stream=0)
    assert len(calls) == 5


def test_binding_checks_workspaces(recorded, monkeypatch):
    """One on another device, or whose elements are not all there (a single one, expanded), would be written out of range."""
    torch, calls, fake = recorded
    record = lambda name: lambda *a: calls.append((name, a)) or 0  # noqa: E731
    monkeypatch.setattr(LQ, "lib", lambda: types.SimpleNamespace(**{n: record(n) for n in (
        "lrqat_qk_rope_bwd", "lrqat_kv_extend", "lrqat_kv_truncate", "lrqat_kv_attn", "lrqat_kv_attn_sinks", "lrqat_kv_attn_shared")}))
    i32, bf = torch.int32, torch.bfloat16
    n = lambda k: fake((k,), i32)  # noqa: E731
    codes, scale = fake((8, 2, 16, 128), torch.int8), fake((8, 2), torch.float32)
    cache, batch = LQ.KVCache.of(codes, codes, scale, scale), LQ.KVBatch.of(n(2), n(3), fake((2, 4), i32), 6, 3, 64)
    blocks, rope = LQ.KVBlocks.of(fake((2, 4), i32), n(64), 16), LQ.QKRope.of(4, 0, 128, None)
    q, g, dg = fake((6, 4, 128), bf), fake((128,), bf), fake((128,), torch.float32)

    def run(ws):
        yield lambda: LQ.kv_attn(cache, batch, q, 1.0, 8, q, ws, stream=0)
        yield lambda: LQ.kv_attn_sinks(cache, batch, q, 1.0, 8, 4, q, ws, stream=0)
        yield lambda: LQ.kv_attn_shared(cache, batch, n(2), 32, q, 1.0, q, ws, stream=0)
        yield lambda: LQ.kv_extend(blocks, n(2), n(2), n(1), n(2), n(1), n(2), n(3), n(5), None, ws, stream=0)
        yield lambda: LQ.kv_truncate(blocks, n(2), n(2), n(1), n(2), n(1), ws, stream=0)
        yield lambda: LQ.qk_rope_bwd(rope, None, q, None, q, None, g, None, q, None, dg, None, False, ws, stream=0)

    good = fake((64,), torch.uint8)
    expanded = types.SimpleNamespace(**{**vars(good), "is_contiguous": torch.zeros(1).expand(64).is_contiguous})
    for call in run(good):
        call()
    assert len(calls) == 6 and all(OK in a and 64 in a for _, a in calls)
    for bad in (fake((64,), torch.uint8, "cuda:1"), fake((64,), torch.uint8, "cpu"), expanded):
        for call in run(bad):
            with pytest.raises(LQ.LrqatError) as e:
                call()
            assert e.value.status == -1
    assert len(calls) == 6


@pytest.mark.parametrize("beyond", [1 << 32, (1 << 32) + 5, 1 << 31, -(1 << 31) - 1, 1 << 70])
def test_binding_refuses_numbers_beyond_32_bits(recorded, monkeypatch, beyond):
    """Their lower 32 bits are another number: 2^32 + 5 sinks would be 5, a window of 2^32 none."""
    torch, _, fake = recorded
    calls = []
    record = lambda *a: calls.append(a) or 0  # noqa: E731
    monkeypatch.setattr(LQ, "_short", None)                        # which leaves such numbers to the long way
    monkeypatch.setattr(LQ, "lib", lambda: types.SimpleNamespace(**{f"lrqat_kv_attn{n}": record for n in (
        "", "_sinks", "_shared", "_workspace_bytes", "_sinks_workspace_bytes", "_shared_workspace_bytes")}))
    i32 = torch.int32
    n = lambda k: fake((k,), i32)  # noqa: E731
    codes, scale, table, q = fake((8, 2, 16, 128), torch.int8), fake((8, 2), torch.float32), fake((2, 4), i32), fake((6, 4, 128), torch.bfloat16)
    cache, batch = LQ.KVCache.of(codes, codes, scale, scale), LQ.KVBatch.of(n(2), n(3), table, 6, 3, 64)

    def run(v):
        yield lambda: LQ.kv_attn(cache, batch, q, 1.0, v, q, None, stream=0)
        yield lambda: LQ.kv_attn_sinks(cache, batch, q, 1.0, v, 4, q, None, stream=0)
        yield lambda: LQ.kv_attn_sinks(cache, batch, q, 1.0, 8, v, q, None, stream=0)
        yield lambda: LQ.kv_attn_shared(cache, batch, n(2), v, q, 1.0, q, None, stream=0)
        yield lambda: LQ.kv_attn_workspace_bytes(cache, batch, 4, v)
        yield lambda: LQ.kv_attn_sinks_workspace_bytes(cache, batch, 4, v, 4)
        yield lambda: LQ.kv_attn_sinks_workspace_bytes(cache, batch, 4, 8, v)
        yield lambda: LQ.kv_attn_shared_workspace_bytes(cache, batch, 4, v)
        yield lambda: LQ.KVBatch.of(n(2), n(3), table, 6, v, 64)
        yield lambda: LQ.KVBatch.of(n(2), n(3), table, 6, 3, v)
        yield lambda: LQ.KVBlocks.of(table, n(64), v, 1)
        yield lambda: LQ.KVBlocks.of(table, n(64), 16, v)
        yield lambda: LQ.QKRope.of(v, 1, 128, None)
        yield lambda: LQ.QKRope.of(1, v, 128, None)
        yield lambda: LQ.QKRope.of(1, 1, v, None)

    for call in run(16):
        call()
    assert len(calls) == 8
    for call in run(beyond):
        with pytest.raises(LQ.LrqatError) as e:
            call()
        assert e.value.status == -1
    assert len(calls) == 8
