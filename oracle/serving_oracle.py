"""Plain numpy float64 definitions of the operators around the quantized linear layer in a block with 8-bit
activations and an 8-bit cache: the fused residual add, root-mean-square norm and per-token quantizer with
its gradient, the paged cache's writes and reads, and attention over it.  Divisions that decide a code, and
stored scales, are fp32, as the interface fixes them.  Imports nothing from the CUDA path."""
from __future__ import annotations

import numpy as np

F64 = np.float64


def rmsnorm(h, gamma, eps):
    """gamma h / sqrt(mean(h^2) + eps), rows of h."""
    h = np.asarray(h, F64)
    return h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * np.asarray(gamma, F64)


def token_scale(y):
    """max|y| / 127 per row, 1 for a row of zeros."""
    a = np.abs(y).max(1)
    return np.where(a > 0, a / 127.0, 1.0)


def rmsnorm_bwd(dy, h, gamma, eps, dh=None):
    """(dx, dgamma) of rmsnorm at h, plus dh in dx; the quantizer behind it is passed straight through."""
    dy, h, gamma = (np.asarray(v, F64) for v in (dy, h, gamma))
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    g = dy * gamma
    dx = r * (g - h * r * r * (g * h).mean(1, keepdims=True))
    return (dx if dh is None else dx + np.asarray(dh, F64)), (dy * h * r).sum(0)


class Cache:
    """One of keys and values: codes [n_blocks, heads, block, d], scale [n_blocks, heads]."""

    def __init__(self, n_blocks, heads, block, d):
        self.codes = np.zeros((n_blocks, heads, block, d), np.int8)
        self.scale = np.full((n_blocks, heads), np.nan, np.float32)
        self.block = block

    def write(self, x, length, blocks):
        """Rows x [n, heads, d] are the newest tokens of a sequence of `length` tokens in `blocks`."""
        x = np.asarray(x, np.float32)
        n = x.shape[0]
        for p0 in range(0, length, self.block):
            new = [p for p in range(p0, min(p0 + self.block, length)) if p >= length - n]
            if not new:
                continue
            blk = blocks[p0 // self.block]
            old = new[0] - p0
            for h in range(x.shape[1]):
                rows = np.stack([x[p - (length - n), h] for p in new])
                a = np.float32(np.abs(rows).max())
                fresh = np.float32(a / np.float32(127.0)) if np.isfinite(a) else np.float32(np.nan)
                was = self.scale[blk, h]
                zeros = was == 0 or (was == 1 and not self.codes[blk, h, :old].any())    # nothing but zeros so far
                if zeros:
                    self.codes[blk, h, :old] = 0
                if old and not zeros:
                    s = was if (was >= fresh or np.isnan(was)) else fresh
                    if s > was:
                        c = self.codes[blk, h, :old].astype(np.float32) * np.float32(was / s)
                        self.codes[blk, h, :old] = np.rint(c).astype(np.int8)
                else:
                    s = np.float32(1.0) if a == 0 else fresh
                self.scale[blk, h] = s
                if np.isnan(s):
                    continue          # the block reads as NaN, whatever its codes are
                for p, row in zip(new, rows):
                    self.codes[blk, h, p - p0] = np.rint(row / s).astype(np.int8)

    def values(self, length, blocks):
        """[length, heads, d] in float64."""
        out = []
        for p in range(length):
            blk = blocks[p // self.block]
            out.append(self.codes[blk, :, p % self.block].astype(F64) * self.scale[blk].astype(F64)[:, None])
        return np.stack(out) if out else np.zeros((0,) + self.codes.shape[1::2], F64)


def attention(q, k, v, length, softmax_scale, window=0):
    """Rows q [n, heads, d] at positions length - n .. length - 1 over k, v [length, kv heads, d].  Returns the
    outputs, sum_j p_j |v_j| (what rounding errors of the probabilities p_j scale with) and the number of keys
    each row sees."""
    q = np.asarray(q, F64)
    n, heads, d = q.shape
    out, mass, seen = np.zeros((n, heads, d)), np.zeros((n, heads, d)), np.zeros(n, int)
    group = heads // max(1, k.shape[1])
    for i in range(n):
        pos = length - n + i
        lo = max(0, pos - window + 1) if window else 0
        if pos < 0:
            continue
        seen[i] = pos + 1 - lo
        for h in range(heads):
            z = softmax_scale * (k[lo:pos + 1, h // group] @ q[i, h])
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, h] = p @ v[lo:pos + 1, h // group]
            mass[i, h] = p @ np.abs(v[lo:pos + 1, h // group])
    return out, mass, seen
