"""The W4A8KV8 attention example end to end against float64 definitions, quantized at the same places.

Tolerance: the outputs pass two bf16 projections (1e-2 each in relative Frobenius norm, the layer's own
tolerance); a code that rounds to the other neighbour moves one element by 1/127 of its row's largest, within it."""
import importlib.util
import os

import numpy as np
import pytest

import oracle as O
from oracle import serving_oracle as SO
from paper_2406_06385_gb300 import lrqat as LQ
from paper_2406_06385_gb300 import workloads as WL

from gpu_util import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("w4a8kv8_attention", os.path.join(ROOT, "examples", "w4a8kv8_attention.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _bf16(x):
    return WL.bf16_to_f32(WL.bf16_bits(np.asarray(x, np.float32))).astype(np.float64)


def _quant(y):
    s = SO.token_scale(y)[:, None]
    return _bf16(np.rint(y / s) * s)


class RefProjection:
    def __init__(self, proj):
        self.L = O.Layer(proj.m, proj.k, proj.r, float(proj.r), 4, 0, WL.PHI_QFIXED, 0)
        self.args = (proj.phi0.cpu().numpy(), proj.s.cpu().numpy(), _np(proj.A).astype(np.float32), _np(proj.B).astype(np.float32))

    def forward(self, x_hat):
        return _bf16(O.linear_fwd(x_hat.astype(np.float32), *self.args, self.L))


@pytest.mark.parametrize("window", [0, 20])
def test_prompts_and_tokens(example, window):
    t = torch()
    t.manual_seed(3)
    hidden, heads, kv_heads, d, block = 256, 4, 2, 64, 16
    qkv, out = example.random_projection((heads + 2 * kv_heads) * d, hidden), example.random_projection(hidden, heads * d)
    g1, g2 = ((1 + 0.2 * t.randn(hidden, device="cuda")).bfloat16() for _ in range(2))
    blk = example.AttentionBlock(qkv, out, g1, g2, heads, kv_heads, d)
    seqs = example.Sequences(3, 128, kv_heads, d, block)
    caches = [SO.Cache(seqs.cache.n_blocks, kv_heads, block, d) for _ in range(2)]
    table = seqs.table.cpu().numpy()
    rq, ro = RefProjection(qkv), RefProjection(out)
    for new in ([37, 1, 70], [1, 1, 1], [1, 4, 1]):
        batch = seqs.append(new)
        x, res = (t.randn(sum(new), hidden, device="cuda").bfloat16() for _ in range(2))
        h, x_hat = blk.step(x, res, seqs.cache, batch, window)
        LQ.get_device_status()
        hr = _np(x) + _np(res)
        y = rq.forward(_quant(SO.rmsnorm(hr, _np(g1), example.EPS))).reshape(-1, heads + 2 * kv_heads, d)
        a, at = np.zeros((sum(new), heads, d)), 0
        for b, n in enumerate(new):
            rows = slice(at, at + n)
            for i, c in enumerate(caches):
                lo = heads + i * kv_heads
                c.write(y[rows, lo:lo + kv_heads], seqs.length[b], table[b])
            k, v = (c.values(seqs.length[b], table[b]) for c in caches)
            a[rows] = SO.attention(y[rows, :heads], k, v, seqs.length[b], 1 / np.sqrt(d), window)[0]
            at += n
        h2 = ro.forward(_quant(_bf16(a).reshape(-1, heads * d))) + _bf16(hr)
        assert O.rel_fro(_np(h), h2) <= 2e-2
        assert O.rel_fro(_np(x_hat), _quant(SO.rmsnorm(h2, _np(g2), example.EPS))) <= 2e-2


def test_training_step(example):
    t = torch()
    t.manual_seed(4)
    T, m, k = 150, 384, 256
    proj = example.random_projection(m, k)
    gamma = (1 + 0.2 * t.randn(k, device="cuda")).bfloat16()
    x, res, dh = (t.randn(T, k, device="cuda").bfloat16() for _ in range(3))
    dy = t.randn(T, m, device="cuda").bfloat16()
    y, dx, dgamma, (dA, dB, ds) = example.train_step(proj, gamma, x, res, dy, dh)
    LQ.get_device_status()
    h = _bf16(_np(x) + _np(res))
    x_hat = _quant(SO.rmsnorm(_np(x) + _np(res), _np(gamma), example.EPS))
    ref = RefProjection(proj)
    g = O.linear_bwd(_np(dy).astype(np.float32), x_hat.astype(np.float32), *ref.args, ref.L)
    dx_ref, dgamma_ref = SO.rmsnorm_bwd(_bf16(g["dX"]), h, _np(gamma), example.EPS, _np(dh))
    assert O.rel_fro(_np(y), ref.forward(x_hat)) <= 1e-2
    assert O.rel_fro(_np(dx), dx_ref) <= 2e-2 and O.rel_fro(_np(dgamma), dgamma_ref) <= 2e-2
    for got, name in ((dA, "dA"), (dB, "dB"), (ds, "ds")):
        assert O.rel_fro(_np(got), g[name]) <= 2e-2, name
