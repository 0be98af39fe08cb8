"""GPU parity of the fused residual add, root-mean-square norm and per-token quantizer, its gradient and the
dequantizer, against float64.

Tolerances: a sum of k squares in fp32 over trees of at most k / threads + 10 additions keeps a relative
error below 1e-5 (half of it after the root); bf16 outputs add half an ulp, 2^-9; a code may differ from
round(y / s) in float64 only where y / s lies within 127 * 1e-5 of a half-integer."""
import numpy as np
import pytest

from oracle import serving_oracle as SO
from paper_2406_06385_gb300 import lrqat as LQ
from paper_2406_06385_gb300 import workloads as WL

from gpu_util import bits_to_f32, empty, to_dev, torch

pytestmark = pytest.mark.gpu

EPS = 1e-5
SHAPES = [(1, 8), (1, 4096), (3, 264), (33, 256), (7, 5120), (400, 1000), (1000, 4096), (5, 8192), (2, 8200),
          (311, 16384)]


def _bf16(a):
    bits = WL.bf16_bits(np.asarray(a, np.float32))
    return bits, WL.bf16_to_f32(bits)


def _inputs(T, k, seed, names):
    rng = np.random.default_rng(seed)
    out = {}
    for n in names:
        if n == "gamma":
            out[n] = _bf16(1 + 0.3 * rng.standard_normal(k))
        else:
            x = rng.standard_normal((T, k)) * 10.0 ** rng.uniform(-2, 2, (T, 1))
            x[:, rng.random(k) < 0.01] *= 20
            out[n] = _bf16(x)
    return out


def _fwd(bits, norm, T, k, residual, out):
    """(H, Y, codes, s) of one call on device copies; `out` names the outputs asked for."""
    t = torch()
    H = empty((T, k), t.int16) if residual else None
    Y = empty((T, k), t.int16) if "Y" in out else None
    q = empty((T, k), t.int8) if "q" in out else None
    s = empty((T,), t.float32) if "s" in out else None
    LQ.add_rmsnorm_fwd(norm, T, to_dev(bits["X"]), to_dev(bits["R"]) if residual else None, to_dev(bits["gamma"]), H, Y, q, s)
    LQ.get_device_status()
    return H, Y, q, s


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("T,k", SHAPES)
def test_forward(T, k, residual):
    d = _inputs(T, k, T + k, ["X", "R", "gamma"])
    bits = {n: v[0] for n, v in d.items()}
    x, r, gamma = (d[n][1].astype(np.float64) for n in ("X", "R", "gamma"))
    h = x + r if residual else x
    y = SO.rmsnorm(h, gamma, EPS)
    norm = LQ.Norm(k, EPS, 8)
    H, Y, q, s = _fwd(bits, norm, T, k, residual, "Yqs")
    if residual:
        assert (np.abs(bits_to_f32(H) - h) <= 2.0 ** -8 * np.abs(h)).all()
    s_ref = SO.token_scale(y)
    s = s.cpu().numpy()
    assert (np.abs(s - s_ref) <= 1e-5 * s_ref).all()
    u = y / s_ref[:, None]
    codes = q.cpu().numpy()
    off = codes != np.rint(u)
    near = np.abs(np.abs(u - np.rint(u)) - 0.5) < 127e-5
    assert not (off & ~near).any() and (np.abs(codes - u) < 0.5 + 127e-5).all()
    # the values are bf16(s c), with one output or both, and from the dequantizer
    values = bits_to_f32(Y)
    assert np.array_equal(values, WL.bf16_to_f32(WL.bf16_bits(codes.astype(np.float32) * s[:, None])))
    assert np.array_equal(values, bits_to_f32(_fwd(bits, norm, T, k, residual, "Y")[1]))
    assert np.array_equal(codes, _fwd(bits, norm, T, k, residual, "qs")[2].cpu().numpy())
    back = empty((T, k), torch().int16)
    LQ.act_dequant(norm, T, to_dev(codes), to_dev(s), back)
    assert np.array_equal(values, bits_to_f32(back))
    # unquantized
    plain = bits_to_f32(_fwd(bits, LQ.Norm(k, EPS, 0), T, k, residual, "Y")[1])
    assert (np.abs(plain - y) <= 2.0 ** -8 * np.abs(y)).all()


def test_rows_of_zeros_and_single_values():
    k = 512
    x = np.zeros((4, k), np.float32)
    x[1, 77] = -3.0
    x[2] = 1e-30
    x[3, :] = 2.0
    bits = {"X": WL.bf16_bits(x), "R": WL.bf16_bits(0 * x), "gamma": WL.bf16_bits(np.ones(k, np.float32))}
    H, Y, q, s = _fwd(bits, LQ.Norm(k, EPS, 8), 4, k, True, "Yqs")
    s, q = s.cpu().numpy(), q.cpu().numpy()
    assert s[0] == 1 and (q[0] == 0).all() and (bits_to_f32(Y)[0] == 0).all()
    assert q[1, 77] == -127 and np.abs(q[1]).sum() == 127
    assert (q[2] == 127).all() and (q[3] == 127).all()
    assert np.array_equal(bits_to_f32(H), WL.bf16_to_f32(bits["X"]))
    # with eps = 0 a row of zeros is 0 / 0
    _, Y, _, s = _fwd(bits, LQ.Norm(k, 0.0, 8), 4, k, True, "Yqs")
    assert np.isnan(s.cpu().numpy()[0]) and np.isnan(bits_to_f32(Y)[0]).all() and s.cpu().numpy()[3] > 0


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_a_value_that_is_not_finite_poisons_its_row_alone(bad):
    T, k = 5, 1024
    d = _inputs(T, k, 3, ["X", "R", "gamma"])
    x = d["X"][1].copy()
    x[2, 1000] = bad
    bits = {"X": WL.bf16_bits(x) if np.isinf(bad) else _nan_bits(d["X"][0], 2, 1000), "R": d["R"][0], "gamma": d["gamma"][0]}
    _, Y, _, s = _fwd(bits, LQ.Norm(k, EPS, 8), T, k, True, "Yqs")
    _, Y0, _, s0 = _fwd({n: v[0] for n, v in d.items()}, LQ.Norm(k, EPS, 8), T, k, True, "Yqs")
    Y, s, Y0, s0 = bits_to_f32(Y), s.cpu().numpy(), bits_to_f32(Y0), s0.cpu().numpy()
    assert np.isnan(s[2]) and np.isnan(Y[2]).all()
    keep = [0, 1, 3, 4]
    assert np.array_equal(s[keep], s0[keep]) and np.array_equal(Y[keep], Y0[keep])


def _nan_bits(bits, i, j):
    out = bits.copy()
    out[i, j] = 0x7FC0
    return out


def test_residual_stream_may_be_written_in_place():
    t = torch()
    T, k = 65, 4096
    d = _inputs(T, k, 9, ["X", "R", "gamma"])
    H, Y, _, _ = _fwd({n: v[0] for n, v in d.items()}, LQ.Norm(k, EPS, 8), T, k, True, "Y")
    R, Y2 = to_dev(d["R"][0]), empty((T, k), t.int16)
    LQ.add_rmsnorm_fwd(LQ.Norm(k, EPS, 8), T, to_dev(d["X"][0]), R, to_dev(d["gamma"][0]), R, Y2, None, None)
    assert t.equal(R, H) and t.equal(Y2, Y)


def _bwd(d, T, k, dh=True, dgamma=None, accumulate=False, want_dgamma=True):
    t = torch()
    norm = LQ.Norm(k, EPS, 8)
    dX = empty((T, k), t.int16)
    if want_dgamma and dgamma is None:
        dgamma = empty((k,), t.float32)
    ws = empty((LQ.add_rmsnorm_bwd_workspace_bytes(norm, T),), t.uint8)
    ws.fill_(0xFF)
    LQ.add_rmsnorm_bwd(norm, T, to_dev(d["dY"][0]), to_dev(d["dH"][0]) if dh else None, to_dev(d["H"][0]),
                       to_dev(d["gamma"][0]), dX, dgamma if want_dgamma else None, accumulate, ws if want_dgamma else None)
    LQ.get_device_status()
    return dX, dgamma


@pytest.mark.parametrize("dh", [True, False])
@pytest.mark.parametrize("T,k", SHAPES)
def test_backward(T, k, dh):
    """dX: half a bf16 ulp and 2^-18 of the terms it is summed from (fp32 with the sums' 1e-5 / 2); dgamma: 1e-5 of
    the sum of magnitudes."""
    d = _inputs(T, k, 2 * T + k, ["dY", "dH", "H", "gamma"])
    dy, dhv, h, gamma = (d[n][1].astype(np.float64) for n in ("dY", "dH", "H", "gamma"))
    dx_ref, dg_ref = SO.rmsnorm_bwd(dy, h, gamma, EPS, dhv if dh else None)
    dX, dgamma = _bwd(d, T, k, dh)
    r = 1 / np.sqrt((h * h).mean(1, keepdims=True) + EPS)
    g = dy * gamma
    terms = r * np.abs(g) + r ** 3 * np.abs(h) * np.abs(g * h).mean(1, keepdims=True) + (np.abs(dhv) if dh else 0)
    assert (np.abs(bits_to_f32(dX) - dx_ref) <= 2.0 ** -8 * np.abs(dx_ref) + 2.0 ** -16 * terms).all()
    assert (np.abs(dgamma.cpu().numpy() - dg_ref) <= 1e-5 * np.abs(dy * h * r).sum(0) + 1e-30).all()
    # a frozen norm gives the same dX, and a second call the same bits
    t = torch()
    assert t.equal(_bwd(d, T, k, dh, want_dgamma=False)[0], dX)
    again = _bwd(d, T, k, dh)
    assert t.equal(again[0], dX) and t.equal(again[1], dgamma)
    # accumulation
    start = np.random.default_rng(1).standard_normal(k).astype(np.float32)
    acc = _bwd(d, T, k, dh, dgamma=to_dev(start), accumulate=True)[1]
    assert np.array_equal(acc.cpu().numpy(), start + dgamma.cpu().numpy())


@pytest.mark.parametrize("T,k", [(70, 4096), (700, 1024)])
def test_gradient_may_be_written_in_place(T, k):
    t = torch()
    d = _inputs(T, k, 13, ["dY", "dH", "H", "gamma"])
    dX, dgamma = _bwd(d, T, k)
    norm = LQ.Norm(k, EPS, 8)
    ws = empty((LQ.add_rmsnorm_bwd_workspace_bytes(norm, T),), t.uint8)
    for over in ("dY", "dH"):
        dev = {n: to_dev(v[0]) for n, v in d.items()}
        again = empty((k,), t.float32)
        LQ.add_rmsnorm_bwd(norm, T, dev["dY"], dev["dH"], dev["H"], dev["gamma"], dev[over], again, False, ws)
        assert t.equal(dev[over], dX) and t.equal(again, dgamma), over


def test_backward_against_differences():
    """<dY, y> changes along a direction v by <dX, v>: central differences of the float64 norm at the bf16 inputs; dX
    in bf16 keeps 2^-9 of each of its elements."""
    T, k = 4, 64
    d = _inputs(T, k, 5, ["dY", "dH", "H", "gamma"])
    dy, h, gamma = (d[n][1].astype(np.float64) for n in ("dY", "H", "gamma"))
    dX, _ = _bwd(d, T, k, dh=False)
    got = bits_to_f32(dX).astype(np.float64)
    rng = np.random.default_rng(6)
    for _ in range(8):
        v = rng.standard_normal((T, k)) * np.abs(h).mean(1, keepdims=True)
        f = lambda e: (SO.rmsnorm(h + e * v, gamma, EPS) * dy).sum()  # noqa: E731
        diff = (f(1e-5) - f(-1e-5)) / 2e-5
        assert abs(diff - (got * v).sum()) <= 2.0 ** -8 * np.abs(got * v).sum() + 1e-6 * np.abs(v).sum()


def test_calls_run_on_the_stream_they_are_given():
    t = torch()
    T, k = 129, 4096
    d = _inputs(T, k, 11, ["X", "R", "gamma"])
    _, Y, _, s = _fwd({n: v[0] for n, v in d.items()}, LQ.Norm(k, EPS, 8), T, k, True, "Yqs")
    X, R, gamma = (to_dev(d[n][0]) for n in ("X", "R", "gamma"))
    H2, Y2, s2 = empty((T, k), t.int16), empty((T, k), t.int16), empty((T,), t.float32)
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    LQ.add_rmsnorm_fwd(LQ.Norm(k, EPS, 8), T, X, R, gamma, H2, Y2, None, s2, stream=side)
    side.synchronize()
    assert t.equal(Y, Y2) and t.equal(s, s2)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("T,k", [(1, 4096), (5, 264), (400, 1000), (7, 5120), (2, 8200)])
def test_a_weight_that_is_not_finite_poisons_every_row(T, k, bad):
    """gamma holds a NaN or an infinity: every row's scale is NaN, so the values, written at once or rebuilt from the
    codes, are NaN alike (0 times infinity included); without the quantizer only that column is lost."""
    t = torch()
    d = _inputs(T, k, 21, ["X", "R", "gamma"])
    j = k - 3
    bits = {n: v[0].copy() for n, v in d.items()}
    bits["gamma"][j] = {True: 0x7FC0, False: 0x7F80 if bad > 0 else 0xFF80}[bool(np.isnan(bad))]
    bits["X"][T - 1, j] = bits["R"][T - 1, j] = 0
    _, Y, q, s = _fwd(bits, LQ.Norm(k, EPS, 8), T, k, True, "Yqs")
    back = empty((T, k), t.int16)
    LQ.act_dequant(LQ.Norm(k, EPS, 8), T, q, s, back)
    assert np.isnan(s.cpu().numpy()).all() and np.isnan(bits_to_f32(Y)).all() and np.isnan(bits_to_f32(back)).all()
    assert np.isnan(_fwd(bits, LQ.Norm(k, EPS, 8), T, k, True, "qs")[3].cpu().numpy()).all()
    plain = bits_to_f32(_fwd(bits, LQ.Norm(k, EPS, 0), T, k, True, "Y")[1])
    assert not np.isfinite(plain[:, j]).any() and np.isfinite(np.delete(plain, j, 1)).all()


def test_codes_of_rows_whose_scale_is_subnormal_keep_their_sign():
    """max|y| of 190 steps of the subnormal range: max|y| / 127 is one step, so y / s reaches 190 and the codes end at
    the 8 bits' ends."""
    k = 256
    x = np.zeros((2, k), np.float32)
    x[0, :4] = 2.0 ** -126 * np.array([1.0, -1.0, 0.5, -0.25])
    x[1] = 1.0
    eps = float(np.float32((2.0 ** 23 / 190) ** 2))          # y = x / sqrt(eps): 190, -190, 95, -47.5 steps of 2^-149
    bits = {"X": WL.bf16_bits(x), "R": None, "gamma": WL.bf16_bits(np.ones(k, np.float32))}
    _, Y, q, s = _fwd(bits, LQ.Norm(k, eps, 8), 2, k, False, "Yqs")
    q, s = q.cpu().numpy(), s.cpu().numpy()
    assert s[0] == np.float32(2.0 ** -149)
    assert q[0, :3].tolist() == [127, -128, 95] and q[0, 3] in (-47, -48) and (q[0, 4:] == 0).all()
    assert (q[1] == 127).all()


@pytest.mark.parametrize("how", ["argument", "current"])
def test_calls_are_queued_behind_the_work_of_their_stream(how):
    """On a side stream some milliseconds of other work and then the copies that fill the inputs: a call on any other
    stream would read what the inputs held before."""
    t = torch()
    T, k = 129, 4096
    d = _inputs(T, k, 22, ["X", "R", "dY", "gamma"])
    norm = LQ.Norm(k, EPS, 8)
    src = {n: to_dev(v[0]) for n, v in d.items()}
    junk, side = empty((1 << 28,), t.float32), t.cuda.Stream()

    def run(dev, stream):
        H, Y, q, s = empty((T, k), t.int16), empty((T, k), t.int16), empty((T, k), t.int8), empty((T,), t.float32)
        dX, dgamma, back = empty((T, k), t.int16), empty((k,), t.float32), empty((T, k), t.int16)
        ws = empty((LQ.add_rmsnorm_bwd_workspace_bytes(norm, T),), t.uint8)
        out = [H, Y, q, s, dX, dgamma, back]
        for o in out:
            o.zero_()
        if stream is not None:
            stream.wait_stream(t.cuda.current_stream())
            with t.cuda.stream(stream):
                for i in range(20):
                    junk.fill_(float(i))
                for n in dev:
                    dev[n].copy_(src[n])
        with t.cuda.stream(stream if how == "current" else None):
            at = stream if how == "argument" else None
            LQ.add_rmsnorm_fwd(norm, T, dev["X"], dev["R"], dev["gamma"], H, Y, q, s, stream=at)
            LQ.act_dequant(norm, T, q, s, back, stream=at)
            LQ.add_rmsnorm_bwd(norm, T, dev["dY"], None, H, dev["gamma"], dX, dgamma, False, ws, stream=at)
        t.cuda.synchronize()
        return out

    want = run(src, None)
    got = run({n: t.zeros_like(v) for n, v in src.items()}, side)
    assert all(t.equal(a, b) for a, b in zip(want, got))
