"""An attention block with 4-bit weights, 8-bit activations and an 8-bit key / value cache (W4A8KV8), as a user
of the library runs it.

Serving, one call per step for a ragged batch of prompts, single tokens or both (kv_attn is faster in two calls, one
for the prompts and one for the single tokens, than over both at once):

    h, x = x + residual, quantized norm       add_rmsnorm_fwd (X_hat per token)
    q, k, v = x W_qkv^T                       linear_fwd_quantized, one fused projection
    cache <- k, v                             kv_write (views of the projection's output)
    a = attention(q, cache)                   kv_attn
    y = quantize(a) W_o^T                     act_quant, linear_fwd_quantized
    h, x = y + h, quantized norm              add_rmsnorm_fwd: what the block's MLP takes

Positions: the block has none of its own.  A model with rotary positions rotates q and k between the projection and
kv_write; the library has no operator for that.

Training, a normed projection that keeps its activations as one byte each: the codes and scales of
add_rmsnorm_fwd, from which act_dequant rebuilds X_hat for the backward of the projection, and
add_rmsnorm_bwd.

    python examples/w4a8kv8_attention.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2406_06385_gb300 import lrqat as LQ  # noqa: E402

EPS = 1e-5


class Projection:
    """A W4 per-channel LR-QAT linear layer [m, k] with per-token 8-bit activations."""

    def __init__(self, W0, A, B):
        (m, k), r = W0.shape, A.shape[1]
        self.m, self.k, self.r = m, k, r
        self.layer = LQ.Layer(m, k, r, float(r), 4, 0, LQ.PHI_QFIXED, 8, None, 1, 0)
        self.s = torch.empty(m, device="cuda")
        self.phi0 = torch.empty(m, k, dtype=torch.int8, device="cuda")
        LQ.range_minmax(self.layer, W0, self.s)
        LQ.downcast(self.layer, W0, self.s, self.phi0)
        self.A, self.B = A, B

    def forward(self, x_hat):
        T = x_hat.shape[0]
        y = torch.empty(T, self.m, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(LQ.fwd_workspace_bytes(self.layer, T), dtype=torch.uint8, device="cuda")
        LQ.linear_fwd_quantized(self.layer, T, x_hat, self.phi0, self.s, self.A, self.B, None, y, ws)
        return y

    def backward(self, dy, x_hat):
        T = x_hat.shape[0]
        dx = torch.empty(T, self.k, dtype=torch.bfloat16, device="cuda")
        dA, dB = torch.empty(self.m, self.r, device="cuda"), torch.empty(self.r, self.k, device="cuda")
        ds = torch.empty(self.m, device="cuda")
        ws = torch.empty(LQ.bwd_workspace_bytes(self.layer, T), dtype=torch.uint8, device="cuda")
        LQ.linear_bwd_quantized(self.layer, T, dy, x_hat, None, self.phi0, self.s, self.A, self.B, None, dx, dA, dB, ds,
                                False, ws)
        return dx, dA, dB, ds


class AttentionBlock:
    def __init__(self, qkv: Projection, out: Projection, gamma_in, gamma_out, heads: int, kv_heads: int, head_dim: int):
        self.qkv, self.out, self.gamma_in, self.gamma_out = qkv, out, gamma_in, gamma_out
        self.heads, self.kv_heads, self.d = heads, kv_heads, head_dim
        self.norm = LQ.Norm(qkv.k, EPS, 8)

    def add_norm(self, x, residual, gamma):
        h, x_hat = torch.empty_like(x), torch.empty_like(x)
        LQ.add_rmsnorm_fwd(self.norm, x.shape[0], x, residual, gamma, h, x_hat, None, None)
        return h, x_hat

    def step(self, x, residual, cache: LQ.KVCache, batch: LQ.KVBatch, window: int = 0):
        """x, residual: bf16 [rows, hidden], the newest tokens of the batch's sequences.  Returns the residual
        stream and the quantized input of the MLP."""
        rows = x.shape[0]
        h, x_hat = self.add_norm(x, residual, self.gamma_in)
        qkv = self.qkv.forward(x_hat).view(rows, self.heads + 2 * self.kv_heads, self.d)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
        LQ.kv_write(cache, batch, k, v)
        a = torch.empty(rows, self.heads, self.d, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(LQ.kv_attn_workspace_bytes(cache, batch, self.heads, window), dtype=torch.uint8, device="cuda")
        LQ.kv_attn(cache, batch, q, 1.0 / math.sqrt(self.d), window, a, ws)
        a_hat = torch.empty_like(a)
        LQ.act_quant(self.out.layer, rows, a, None, a_hat)
        return self.add_norm(self.out.forward(a_hat.view(rows, -1)), h, self.gamma_out)


class Sequences:
    """A pool of cache blocks and the sequences in it."""

    def __init__(self, n_seqs: int, max_len: int, kv_heads: int, head_dim: int, block: int):
        self.block, width = block, -(-max_len // block)
        shape = (n_seqs * width, kv_heads, block, head_dim)
        codes = [torch.empty(shape, dtype=torch.int8, device="cuda") for _ in range(2)]
        scale = [torch.empty(shape[:2], device="cuda") for _ in range(2)]
        self.cache = LQ.KVCache.of(*codes, *scale)
        self.table = torch.randperm(n_seqs * width, device="cuda").int().view(n_seqs, width)
        self.length = [0] * n_seqs

    def append(self, new):
        """The batch that adds new[b] tokens to sequence b."""
        self.length = [n + m for n, m in zip(self.length, new)]
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        as_int = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        return LQ.KVBatch.of(as_int(self.length), as_int(starts), self.table, starts[-1], max(new), max(self.length))


def train_step(proj: Projection, gamma, x, residual, dy, dh):
    """Forward and backward of a normed projection.  Between the two it keeps one byte and, per token, one scale of
    the projection's input.  Returns y, the gradients of x (and residual) and gamma, and the projection's."""
    T, k = x.shape
    norm = LQ.Norm(k, EPS, 8)
    h, x_hat = torch.empty_like(x), torch.empty_like(x)
    codes, s = torch.empty(T, k, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    LQ.add_rmsnorm_fwd(norm, T, x, residual, gamma, h, x_hat, codes, s)
    y = proj.forward(x_hat)
    del x_hat                                            # the backward rebuilds it
    x_hat = torch.empty_like(x)
    LQ.act_dequant(norm, T, codes, s, x_hat)
    dx_hat, dA, dB, ds = proj.backward(dy, x_hat)
    dx, dgamma = torch.empty_like(x), torch.empty(k, device="cuda")
    ws = torch.empty(LQ.add_rmsnorm_bwd_workspace_bytes(norm, T), dtype=torch.uint8, device="cuda")
    LQ.add_rmsnorm_bwd(norm, T, dx_hat, dh, h, gamma, dx, dgamma, False, ws)
    return y, dx, dgamma, (dA, dB, ds)


def random_projection(m: int, k: int, r: int = 8):
    return Projection(torch.randn(m, k, device="cuda") / math.sqrt(k), (torch.randn(m, r, device="cuda") / 64).bfloat16(),
                      (torch.randn(r, k, device="cuda") * 1e-2).bfloat16())


def main():
    torch.manual_seed(0)
    hidden, heads, kv_heads, d = 4096, 32, 8, 128
    block = AttentionBlock(random_projection((heads + 2 * kv_heads) * d, hidden), random_projection(hidden, heads * d),
                           torch.ones(hidden, device="cuda").bfloat16(), torch.ones(hidden, device="cuda").bfloat16(),
                           heads, kv_heads, d)
    seqs = Sequences(4, 1024, kv_heads, d, 64)
    for new in ([700, 33, 1, 256], [1, 1, 1, 1], [1, 1, 5, 1]):       # prompts, a token each, drafted tokens for one
        batch = seqs.append(new)
        x, residual = (torch.randn(sum(new), hidden, device="cuda").bfloat16() for _ in range(2))
        h, x_hat = block.step(x, residual, seqs.cache, batch)
        LQ.get_device_status()
        print(f"new tokens {new}: residual stream rms {h.float().pow(2).mean().sqrt():.3f}, "
              f"MLP input rms {x_hat.float().pow(2).mean().sqrt():.3f}")
    T = 1000
    x, residual, dh = (torch.randn(T, hidden, device="cuda").bfloat16() for _ in range(3))
    dy = torch.randn(T, hidden, device="cuda").bfloat16()
    y, dx, dgamma, _ = train_step(random_projection(hidden, hidden), block.gamma_in, x, residual, dy, dh)
    LQ.get_device_status()
    print(f"training step: y rms {y.float().pow(2).mean().sqrt():.3f}, dx rms {dx.float().pow(2).mean().sqrt():.3f}, "
          f"dgamma rms {dgamma.pow(2).mean().sqrt():.3f}")


if __name__ == "__main__":
    main()
