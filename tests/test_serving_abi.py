"""The norm, cache and attention entry points reject bad arguments on the host before any CUDA work."""
import ctypes
import types

import pytest

from paper_2406_06385_gb300 import lrqat as LQ
from paper_2406_06385_gb300.build import build

OK = 16   # a 16-byte aligned address that is never followed


@pytest.fixture(scope="module")
def lib():
    build()
    return LQ.lib()


def _norm(**kw):
    return LQ.Norm(**dict(dict(k=256, eps=1e-5, act_bits=8), **kw))


def _fwd(lib, norm, T=4, X=OK, R=OK, gamma=OK, H=OK, Y=OK, Y_q=OK, s=OK):
    return lib.lrqat_add_rmsnorm_fwd(ctypes.byref(norm), T, X, R, gamma, H, Y, Y_q, s, None)


@pytest.mark.parametrize("kw,status", [(dict(k=0), -1), (dict(k=12), -2), (dict(k=16392), -2), (dict(eps=-1.0), -1),
                                       (dict(eps=float("nan")), -1), (dict(act_bits=4), -2)])
def test_norm_settings(lib, kw, status):
    assert _fwd(lib, _norm(**kw)) == status and LQ.last_error()
    assert lib.lrqat_act_dequant(ctypes.byref(_norm(**kw)), 4, OK, OK, OK, None) == status
    assert lib.lrqat_add_rmsnorm_bwd(ctypes.byref(_norm(**kw)), 4, OK, OK, OK, OK, OK, None, 0, None, 0, None) == status
    assert lib.lrqat_add_rmsnorm_bwd_workspace_bytes(ctypes.byref(_norm(**kw)), 4) == 0


def test_norm_pointers(lib):
    n = _norm()
    assert _fwd(lib, n, T=0) == -1
    for name in ("X", "gamma", "H"):
        assert _fwd(lib, n, **{name: None}) == -1, name
    for name in ("X", "R", "gamma", "H", "Y", "Y_q", "s"):
        assert _fwd(lib, n, **{name: 24}) == -3, name
    assert _fwd(lib, n, Y=None, Y_q=None) == -1
    assert _fwd(lib, n, s=None) == -1
    assert _fwd(lib, _norm(act_bits=0)) == -1                     # codes of an unquantized norm
    bwd = lambda dgamma, ws, size: lib.lrqat_add_rmsnorm_bwd(  # noqa: E731
        ctypes.byref(n), 64, OK, None, OK, OK, OK, dgamma, 0, ws, size, None)
    need = lib.lrqat_add_rmsnorm_bwd_workspace_bytes(ctypes.byref(n), 64)
    assert need > 0 and bwd(OK, None, need) == -4 and bwd(OK, OK, need - 1) == -4 and bwd(24, OK, need) == -3
    assert bwd(OK, 24, need) == -3
    assert lib.lrqat_act_dequant(ctypes.byref(n), 4, OK, None, OK, None) == -1


def _cache(**kw):
    return LQ.KVCache(**dict(dict(n_blocks=8, n_kv_heads=2, head_dim=128, block=16, k_codes=OK, v_codes=OK,
                                  k_scale=OK, v_scale=OK), **kw))


def _batch(**kw):
    return LQ.KVBatch(**dict(dict(n_seqs=2, max_blocks=4, len=OK, row_start=OK, block_table=OK, rows=6, max_rows=3,
                                  max_len=64), **kw))


def _calls(lib, c, b, x=OK, ld=256, heads=4, ldq=512, scale=1.0, window=0, ws=OK, size=1 << 30):
    c, b = ctypes.byref(c), ctypes.byref(b)
    return [lambda: lib.lrqat_kv_write(c, b, x, ld, OK, 256, None), lambda: lib.lrqat_kv_read(c, b, OK, 256, x, ld, None),
            lambda: lib.lrqat_kv_attn(c, b, heads, scale, window, x, ldq, OK, 512, ws, size, None)]


@pytest.mark.parametrize("kw,status", [
    (dict(n_blocks=0), -1), (dict(n_kv_heads=0), -1), (dict(head_dim=96), -2), (dict(block=8), -2), (dict(block=48), -2),
    (dict(k_codes=None), -1), (dict(v_scale=None), -1), (dict(v_codes=24), -3), (dict(k_scale=8), -3)])
def test_cache_settings(lib, kw, status):
    for call in _calls(lib, _cache(**kw), _batch()):
        assert call() == status and LQ.last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(n_seqs=0), -1), (dict(n_seqs=65536), -2), (dict(max_blocks=0), -1), (dict(rows=-1), -1), (dict(max_rows=-1), -1),
    (dict(max_len=-1), -1), (dict(max_len=65), -1), (dict(max_blocks=1 << 28), -2), (dict(len=None), -1),
    (dict(row_start=None), -1), (dict(block_table=None), -1), (dict(len=18), -3), (dict(rows=1 << 31), -2)])
def test_batch_settings(lib, kw, status):
    for call in _calls(lib, _cache(), _batch(**kw)):
        assert call() == status and LQ.last_error()


def test_row_arrays(lib):
    for call in _calls(lib, _cache(), _batch(), x=None, ldq=512):
        assert call() == -1
    for call in _calls(lib, _cache(), _batch(), x=24):
        assert call() == -3
    for call in _calls(lib, _cache(), _batch(), ld=248, ldq=504):
        assert call() == -1                                       # rows closer together than a row is long
    for call in _calls(lib, _cache(), _batch(), ld=257, ldq=513):
        assert call() == -3
    # a batch without rows is no work
    for call in _calls(lib, _cache(), _batch(rows=0)):
        assert call() == 0


def test_attention_settings(lib):
    attn = lambda c=None, b=None, **kw: _calls(lib, c or _cache(), b or _batch(), **kw)[2]()  # noqa: E731
    assert attn(heads=0) == -1 and attn(heads=3) == -1
    assert attn(window=-1) == -1
    assert attn(scale=float("inf")) == -1 and attn(scale=float("nan")) == -1
    long = _batch(max_blocks=4096, max_len=65536)
    need = lib.lrqat_kv_attn_workspace_bytes(ctypes.byref(_cache()), ctypes.byref(long), 4, 0)
    assert need > 0
    assert attn(b=long, ws=None, size=need) == -4 and attn(b=long, size=need - 1) == -4
    assert attn(b=long, ws=24, size=need) == -3
    assert lib.lrqat_kv_attn_workspace_bytes(ctypes.byref(_cache()), ctypes.byref(long), 3, 0) == 0


def test_binding_checks_tensor_layouts():
    torch = pytest.importorskip("torch")
    k = torch.zeros(4, 2, 16, 64, dtype=torch.int8)
    s = torch.zeros(4, 2)
    assert LQ.KVCache.of(k, k, s, s).block == 16
    for bad in ((k, k[:3], s, s), (k, k, s[:, :1], s), (k.transpose(1, 2), k, s, s)):
        with pytest.raises(LQ.LrqatError):
            LQ.KVCache.of(*bad)
    n, t = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.int32)
    with pytest.raises(LQ.LrqatError):
        LQ.KVBatch.of(n, n, t, 3, 1, 16)
    with pytest.raises(LQ.LrqatError):
        LQ._rows(torch.zeros(3, 2, 64).transpose(0, 1), 3, 64)
    assert LQ._rows(torch.zeros(3, 6, 64)[:, :2], 2, 64) == 384


def test_binding_checks_types_and_devices_of_caches_and_batches():
    """A whole number is int64 in torch unless asked otherwise: as a block table it would be read as id, 0, id, 0."""
    torch = pytest.importorskip("torch")
    k, s = torch.zeros(4, 2, 16, 64, dtype=torch.int8), torch.zeros(4, 2)
    LQ.KVCache.of(k, k, s, s)
    for bad in ((k.to(torch.uint8), k, s, s), (k, k.float(), s, s), (k, k.int(), s, s), (k, k, s.double(), s),
                (k, k, s, s.half()), (k, k, s, s.int()), (k, k.to("meta"), s, s), (k, k, s, s.to("meta"))):
        with pytest.raises(LQ.LrqatError) as e:
            LQ.KVCache.of(*bad)
        assert e.value.status == -1
    arrays = [torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.int32)]
    LQ.KVBatch.of(*arrays, 3, 1, 16)
    for i in range(3):
        for bad in (arrays[i].long(), arrays[i].float(), arrays[i].short(), arrays[i].to("meta")):
            with pytest.raises(LQ.LrqatError) as e:
                LQ.KVBatch.of(*arrays[:i], bad, *arrays[i + 1:], 3, 1, 16)
            assert e.value.status == -1


def _stand_in(torch, shape, dtype, device="cuda:0"):
    """What the binding asks of a tensor, with an address that is never followed."""
    t = torch.zeros(shape, dtype=dtype)
    return types.SimpleNamespace(shape=t.shape, dtype=dtype, stride=t.stride, numel=t.numel, element_size=t.element_size,
                                 is_contiguous=lambda: True, is_cuda=device != "cpu",
                                 device=torch.device(device), data_ptr=lambda: OK,
                                 get_device=lambda: -1 if device == "cpu" else int(device[5:]))


def test_binding_checks_row_arrays(monkeypatch):
    """Row arrays shorter than the batch (read or written out of range on the device), of another type, or elsewhere
    than the cache are refused before the library is called."""
    torch = pytest.importorskip("torch")
    calls = []
    record = lambda name: lambda *a: calls.append(name) or 0  # noqa: E731
    monkeypatch.setattr(LQ, "lib", lambda: types.SimpleNamespace(
        **{n: record(n) for n in ("lrqat_kv_write", "lrqat_kv_read", "lrqat_kv_attn")}))
    fake = lambda shape, dtype, device="cuda:0": _stand_in(torch, shape, dtype, device)  # noqa: E731

    def objects(device="cuda:0"):
        codes, scale = fake((8, 2, 16, 128), torch.int8, device), fake((8, 2), torch.float32, device)
        i32 = lambda *shape: fake(shape, torch.int32, device)  # noqa: E731
        return LQ.KVCache.of(codes, codes, scale, scale), LQ.KVBatch.of(i32(2), i32(3), i32(2, 4), 6, 3, 64)

    cache, batch = objects()
    ws = fake((64,), torch.uint8)

    def run(kv, kv2, q, o, ws=ws, cache=cache, batch=batch):
        for f in (lambda: LQ.kv_write(cache, batch, kv, kv2, stream=0), lambda: LQ.kv_read(cache, batch, kv, kv2, stream=0),
                  lambda: LQ.kv_attn(cache, batch, q, 1.0, 0, o, ws, stream=0)):
            yield f

    kv, q = fake((6, 2, 128), torch.bfloat16), fake((6, 4, 128), torch.int16)
    for f in run(kv, kv, q, q):
        f()
    for f in run(fake((7, 2, 128), torch.int16), kv, q, fake((9, 4, 128), torch.bfloat16)):    # longer ones are fine
        f()
    for f in run(kv, kv, q, q, None, LQ.KVCache(8, 2, 128, 16, OK, OK, OK, OK), LQ.KVBatch(2, 4, OK, OK, OK, 6, 3, 64)):
        f()
    assert len(calls) == 9
    bad = lambda **kw: (fake(**{**dict(shape=(6, 2, 128), dtype=torch.bfloat16), **kw}),  # noqa: E731
                        fake(**{**dict(shape=(6, 4, 128), dtype=torch.bfloat16), **kw, **(
                            {"shape": (kw["shape"][0], 4, 128)} if "shape" in kw else {})}))
    for kw in (dict(shape=(5, 2, 128)), dict(shape=(0, 2, 128)), dict(dtype=torch.float16), dict(dtype=torch.float32),
               dict(device="cpu"), dict(device="cuda:1")):
        bkv, bq = bad(**kw)
        for args in ((bkv, kv, bq, q), (kv, bkv, q, bq)):
            for f in run(*args):
                with pytest.raises(LQ.LrqatError) as e:
                    f()
                assert e.value.status == -1
    with pytest.raises(LQ.LrqatError):
        LQ.kv_attn(cache, batch, q, 1.0, 0, q, fake((64,), torch.uint8, "cpu"), stream=0)
    for pair in ((objects("cpu")[0], batch), (cache, objects("cpu")[1])):
        for f in run(kv, kv, q, q, None, *pair):
            with pytest.raises(LQ.LrqatError):
                f()
    assert len(calls) == 9


def test_binding_takes_a_single_row_of_any_stride():
    torch = pytest.importorskip("torch")
    row = torch.zeros(3, 517)[:, :256].unflatten(1, (2, 128))[1:2]
    assert row.stride()[0] == 517
    assert LQ._rows(row, 2, 128) == 256                       # 517 is no multiple of 8, and nothing lies at it
    assert LQ._rows(row.expand(1, 2, 128), 2, 128) == 256
    assert LQ._rows(torch.zeros(0, 2, 128), 2, 128) == 256


@pytest.mark.parametrize("missing", ["_cuda_getDevice", "_cuda_getCurrentRawStream"])
def test_the_current_stream_does_not_hang_on_private_names(monkeypatch, missing):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(LQ, "_current_stream", None, raising=False)
    monkeypatch.delattr(torch._C, missing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=4096))
    assert LQ._stream(None) == 4096
    assert LQ._stream(types.SimpleNamespace(cuda_stream=32)) == 32 and LQ._stream(48) == 48
