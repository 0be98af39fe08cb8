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


def attention(q, k, v, length, softmax_scale, window=0, sinks=0):
    """Rows q [n, heads, d] at positions length - n .. length - 1 over k, v [length, kv heads, d], through a window that
    leaves the first `sinks` keys visible.  Returns the outputs, sum_j p_j |v_j| (what rounding errors of the
    probabilities p_j scale with) and the number of keys each row sees."""
    q = np.asarray(q, F64)
    n, heads, d = q.shape
    out, mass, seen = np.zeros((n, heads, d)), np.zeros((n, heads, d)), np.zeros(n, int)
    group = heads // max(1, k.shape[1])
    for i in range(n):
        pos = length - n + i
        if pos < 0:
            continue
        lo = max(0, pos - window + 1) if window else 0
        keys = np.r_[0:min(lo, sinks), lo:pos + 1]
        seen[i] = len(keys)
        for h in range(heads):
            z = softmax_scale * (k[keys, h // group] @ q[i, h])
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, h] = p @ v[keys, h // group]
            mass[i, h] = p @ np.abs(v[keys, h // group])
    return out, mass, seen


def rotate(x, pos, freq, neighbours=False, back=False):
    """Rows x [n, heads, d] at positions pos [n]: pair i of the first 2 len(freq) elements of each head turned by the
    angle pos freq[i] (by its negative where `back`)."""
    x = np.array(x, F64)
    rot = 2 * len(freq)
    # the angle modulo a turn in extended precision: positions reach 2^31
    w = np.asarray(pos, np.longdouble)[:, None] * np.asarray(freq, np.longdouble)[None]
    w = np.remainder(w, 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(F64)[:, None]
    c, s = np.cos(w), np.sin(w) * (-1 if back else 1)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if neighbours else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * c - b * s, a * s + b * c
    if neighbours:
        x[..., 0:rot:2], x[..., 1:rot:2] = a, b
    else:
        x[..., :rot // 2], x[..., rot // 2:rot] = a, b
    return x


def head_norm_rope(x, gamma, pos, freq, eps, neighbours=False):
    """Norm of each head of x [n, heads, d] (none where gamma is None), then its rotation."""
    x = np.asarray(x, F64)
    if gamma is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gamma, F64)
    return rotate(x, pos, freq, neighbours)


def head_norm_rope_bwd(dy, x, gamma, pos, freq, eps, neighbours=False):
    """(dx, dgamma) of head_norm_rope at x; dgamma is None where gamma is."""
    g = rotate(dy, pos, freq, neighbours, back=True)
    if gamma is None:
        return g, None
    x, gamma = np.asarray(x, F64), np.asarray(gamma, F64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dx = r * (g * gamma - x * r * r * (g * gamma * x).mean(-1, keepdims=True))
    return dx, (g * x * r).sum((0, 1))


class Blocks:
    """Tables [n_seqs][max_blocks] and the list of free blocks; `len` per sequence."""

    def __init__(self, table, free_ids, free, length, block, pinned=0):
        self.table, self.free_ids = np.array(table, np.int32), np.array(free_ids, np.int32)
        self.free, self.len, self.block, self.pinned = int(free), [int(n) for n in length], block, pinned

    def extend(self, add, rows):
        """(batch lengths, row starts, positions, slots, whether a sequence was refused)."""
        P, most = self.block, self.table.shape[1] * self.block
        start, batch_len, pos, slot = [0], [], [-1] * rows, [-1] * rows
        ok_all, dry, free = True, False, self.free if 0 <= self.free <= len(self.free_ids) else 0
        ok_all = free == self.free
        for b, a in enumerate(int(a) for a in add):
            r0, n = start[-1], self.len[b]
            start.append(r0 + abs(a))
            ok = 0 <= n <= most and n + max(a, 0) <= most and start[-1] <= rows
            new = [c for c in range(self.pinned, -(-(n + a) // P)) if c * P >= n] if ok and a > 0 else []
            if new and (dry or len(new) > free):
                ok, dry = False, True
            ok_all &= ok
            batch_len.append(n + a if ok and a >= 0 else 0)
            if not ok or a <= 0:
                continue
            for c in new:
                free -= 1
                self.table[b, c] = self.free_ids[free]
            for i in range(a):
                pos[r0 + i] = n + i
                slot[r0 + i] = int(self.table[b, (n + i) // P]) * P + (n + i) % P
            self.len[b] = n + a
        if 0 <= self.free <= len(self.free_ids):
            self.free = free
        return batch_len, [min(r, 2 ** 31 - 1) for r in start], pos, slot, not ok_all

    def truncate(self, keep):
        """Whether a sequence was refused."""
        P, most, known = self.block, self.table.shape[1] * self.block, 0 <= self.free <= len(self.free_ids)
        back, full, ok_all = [], False, known
        for b, k in enumerate(int(k) for k in keep):
            n = self.len[b]
            k = min(n, max(k, 0))
            if not 0 <= n <= most:
                ok_all = False
                continue
            gone = [int(self.table[b, c]) for c in range(max(-(-k // P), self.pinned), -(-n // P))]
            if gone and (full or not known or self.free + len(back) + len(gone) > len(self.free_ids)):
                ok_all, full = False, True
                continue
            back += gone
            self.len[b] = k
        self.free_ids[self.free:self.free + len(back)] = back[::-1]
        self.free += len(back)
        return not ok_all
