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

With rotary positions, q and k are normed by head and rotated in place between the projection and kv_write
(qk_rope_fwd); the attention may leave a few first tokens visible behind its window (kv_attn_sinks) or read a prefix that
all sequences share once for all of them (kv_attn_shared).  RunningSequences keeps lengths, block tables and the list of free
blocks on the device (kv_extend, kv_truncate), so that a step copies nothing but how many tokens each sequence gets.

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
    def __init__(self, qkv: Projection, out: Projection, gamma_in, gamma_out, heads: int, kv_heads: int, head_dim: int,
                 rope: LQ.QKRope = None, gamma_q=None, gamma_k=None):
        self.qkv, self.out, self.gamma_in, self.gamma_out = qkv, out, gamma_in, gamma_out
        self.rope, self.gamma_q, self.gamma_k = rope, gamma_q, gamma_k
        self.heads, self.kv_heads, self.d = heads, kv_heads, head_dim
        self.norm = LQ.Norm(qkv.k, EPS, 8)

    def add_norm(self, x, residual, gamma):
        h, x_hat = torch.empty_like(x), torch.empty_like(x)
        LQ.add_rmsnorm_fwd(self.norm, x.shape[0], x, residual, gamma, h, x_hat, None, None)
        return h, x_hat

    def step(self, x, residual, cache: LQ.KVCache, batch: LQ.KVBatch, window: int = 0, sinks: int = 0, pos=None,
             prefix_table=None):
        """x, residual: bf16 [rows, hidden], the newest tokens of the batch's sequences; pos: their positions, for a
        block with a rotation; prefix_table: the cache blocks that all sequences start with.  Returns the residual
        stream and the quantized input of the MLP."""
        rows = x.shape[0]
        h, x_hat = self.add_norm(x, residual, self.gamma_in)
        qkv = self.qkv.forward(x_hat).view(rows, self.heads + 2 * self.kv_heads, self.d)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
        if self.rope is not None:
            LQ.qk_rope_fwd(self.rope, pos, q, k, self.gamma_q, self.gamma_k, q, k)
        LQ.kv_write(cache, batch, k, v)
        a, scale = torch.empty(rows, self.heads, self.d, dtype=torch.bfloat16, device="cuda"), 1.0 / math.sqrt(self.d)
        room = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        if prefix_table is not None:
            prefix = prefix_table.numel() * cache.block
            ws = room(LQ.kv_attn_shared_workspace_bytes(cache, batch, self.heads, prefix))
            LQ.kv_attn_shared(cache, batch, prefix_table, prefix, q, scale, a, ws)
        elif sinks:
            ws = room(LQ.kv_attn_sinks_workspace_bytes(cache, batch, self.heads, window, sinks))
            LQ.kv_attn_sinks(cache, batch, q, scale, window, sinks, a, ws)
        else:
            ws = room(LQ.kv_attn_workspace_bytes(cache, batch, self.heads, window))
            LQ.kv_attn(cache, batch, q, scale, window, a, ws)
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


class RunningSequences:
    """The same with everything on the device; the first `prefix_blocks` blocks are a prefix of all sequences."""

    def __init__(self, n_seqs: int, max_len: int, n_blocks: int, kv_heads: int, head_dim: int, block: int, prefix_blocks: int = 0):
        shape, width = (n_blocks, kv_heads, block, head_dim), -(-max_len // block)
        codes = [torch.empty(shape, dtype=torch.int8, device="cuda") for _ in range(2)]
        scale = [torch.empty(shape[:2], device="cuda") for _ in range(2)]
        self.cache = LQ.KVCache.of(*codes, *scale)
        ints = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")  # noqa: E731
        ids = torch.randperm(n_blocks, device="cuda").int()
        self.prefix_table = ids[n_blocks - prefix_blocks:].clone()
        self.free = torch.full((1,), n_blocks - prefix_blocks, dtype=torch.int32, device="cuda")
        self.table = ints(n_seqs, width)
        self.table[:, :prefix_blocks] = self.prefix_table
        self.length = ints(n_seqs)
        self.blocks = LQ.KVBlocks.of(self.table, ids, block, prefix_blocks)
        self.batch_len, self.start, self.max_len = ints(n_seqs), ints(n_seqs + 1), max_len
        self.room = torch.empty(LQ.kv_blocks_workspace_bytes(self.blocks), dtype=torch.uint8, device="cuda")

    def append(self, new, rows: int, max_new: int):
        """The batch that adds new[b] tokens (int32 on the device; below 0: rows of padding) to sequence b, and the positions
        of its rows; rows, max_new: bounds on all rows and on a sequence's."""
        pos = torch.empty(rows, dtype=torch.int32, device="cuda")
        LQ.kv_extend(self.blocks, self.length, new, self.free, self.length, self.free, self.batch_len, self.start, pos, None,
                     self.room)
        return LQ.KVBatch.of(self.batch_len, self.start, self.table, rows, max_new, self.max_len), pos

    def shorten(self, keep):
        """Sequence b to keep[b] tokens (0: it is finished)."""
        LQ.kv_truncate(self.blocks, self.length, keep, self.free, self.length, self.free, self.room)


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
    # the same with rotary positions, behind a prefix of 512 tokens that is in the cache once
    block.rope = LQ.QKRope.of(heads, kv_heads, d, LQ.rope_turns([10000.0 ** (-2 * i / d) for i in range(d // 2)]).cuda())
    running = RunningSequences(4, 2048, 128, kv_heads, d, 64, prefix_blocks=8)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    rows = lambda n: [torch.randn(n, hidden, device="cuda").bfloat16() for _ in range(2)]  # noqa: E731
    alone = LQ.KVBatch.of(ints([512]), ints([0, 512]), running.prefix_table[None], 512, 512, 512)
    block.step(*rows(512), running.cache, alone, pos=torch.arange(512, device="cuda").int())
    running.length.fill_(512)
    for new, keep in (([40, 7, 90, 1], None), ([4, 4, 4, -1], [1, 1, 2, 1]), ([1, 1, 1, 1], None)):
        n = sum(abs(m) for m in new)
        batch, pos = running.append(ints(new), n, max(new))
        h, x_hat = block.step(*rows(n), running.cache, batch, pos=pos, prefix_table=running.prefix_table)
        if keep:                                                     # the drafted tokens that were wrong
            running.shorten(running.length - ints([max(m - k, 0) for m, k in zip(new, keep)]))
        LQ.get_device_status()
        print(f"shared prefix, new tokens {new}: MLP input rms {x_hat.float().pow(2).mean().sqrt():.3f}, "
              f"lengths {running.length.tolist()}, free blocks {int(running.free)}")
    T = 1000
    x, residual, dh = (torch.randn(T, hidden, device="cuda").bfloat16() for _ in range(3))
    dy = torch.randn(T, hidden, device="cuda").bfloat16()
    y, dx, dgamma, _ = train_step(random_projection(hidden, hidden), block.gamma_in, x, residual, dy, dh)
    LQ.get_device_status()
    print(f"training step: y rms {y.float().pow(2).mean().sqrt():.3f}, dx rms {dx.float().pow(2).mean().sqrt():.3f}, "
          f"dgamma rms {dgamma.pow(2).mean().sqrt():.3f}")


if __name__ == "__main__":
    main()
