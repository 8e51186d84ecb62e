"""Plain 64-bit reference of the 8-bit KV cache, its attention and the norm and
rotation of query and key heads (test infrastructure)."""

import numpy as np
import torch

BLOCK = 64
FLUSH = 2.0 ** -90


def round_to(x, dtype):
    """float64 numpy -> the nearest values of a storage dtype, as float64."""
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(t).double().numpy()


def scale_of(values, fmt):
    """The scale of a block's values (any shape, float64)."""
    if not np.all(np.isfinite(values)):
        return np.float32(np.nan)
    amax = float(np.abs(values).max()) if values.size else 0.0
    if amax < FLUSH:
        return np.float32(0)
    if fmt == "int8":
        return np.float32(np.float32(amax) / np.float32(127))
    e = -160
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return np.float32(2.0 ** e)


def nearest(y, fmt):
    """float64 -> the nearest numbers of the format, ties to even.  The quotient of two fp32 numbers is never within
    2^-33 of a tie without being one, so float64's own rounding decides nothing."""
    if fmt == "int8":
        return np.rint(y)
    a = np.abs(y)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -40)))
    e = np.where(2.0 ** e > a, e - 1, e)
    step = 2.0 ** (np.maximum(e, -6) - 3)
    return np.rint(y / step) * step


def to_bytes(numbers, fmt):
    t = torch.from_numpy(np.ascontiguousarray(numbers, dtype=np.float32))
    t = t.to(torch.int8) if fmt == "int8" else t.to(torch.float8_e4m3fn)
    return t.view(torch.uint8).numpy()


def from_bytes(codes, fmt):
    t = torch.from_numpy(np.ascontiguousarray(codes))
    t = t.view(torch.int8) if fmt == "int8" else t.view(torch.float8_e4m3fn)
    return t.to(torch.float32).double().numpy()


def offsets(side, dh):
    """Byte of element (t, d) in a block."""
    t, d = np.arange(BLOCK)[:, None], np.arange(dh)[None, :]
    if side == "k":
        return (t // 16) * 16 * dh + (d // 64) * 1024 + ((d % 64) // 16) * 256 + (t % 16) * 16 + d % 16
    return (d // 16) * 1024 + ((t % 16) // 4) * 256 + (d % 16) * 16 + (t % 4) * 4 + t // 16


class RefCache:
    """Codes [B, H, T, 64 dh] (as stored) and scales [B, H, T] of both sides."""

    def __init__(self, fmt, B, H, dh, capacity, rng=None):
        T = (capacity + BLOCK - 1) // BLOCK
        self.fmt, self.B, self.H, self.dh, self.cap = fmt, B, H, dh, capacity
        self.codes, self.scales = {}, {}
        for s in "kv":
            self.codes[s] = np.zeros((B, H, T, BLOCK * dh), np.uint8)
            self.scales[s] = np.zeros((B, H, T), np.float32)
            if rng is not None:                     # what memory may hold before it is written: any bytes
                self.codes[s][:] = rng.integers(0, 256, self.codes[s].shape, dtype=np.uint8)
                self.scales[s][:] = rng.standard_normal(self.scales[s].shape)

    def block(self, s, b, h, t):
        """Numbers [64, dh] of a block, before the scale."""
        return from_bytes(self.codes[s][b, h, t][offsets(s, self.dh)], self.fmt)

    def write(self, rows, first, count):
        """rows {"k": [B, n, H dh], "v": ...} float64; sequence b's first count[b] as tokens first[b] + i."""
        for b in range(self.B):
            f, n = int(first[b]), int(np.clip(count[b], 0, rows["k"].shape[1]))
            if n == 0 or f < 0 or f + n > self.cap:
                continue
            for t in range(f // BLOCK, (f + n - 1) // BLOCK + 1):
                lo, hi = max(f - t * BLOCK, 0), min(f + n - t * BLOCK, BLOCK)
                for s in "kv":
                    new = rows[s][b, t * BLOCK + lo - f:t * BLOCK + hi - f].reshape(hi - lo, self.H, self.dh)
                    for h in range(self.H):
                        self._write(s, b, h, t, lo, hi, new[:, h])

    def _write(self, s, b, h, t, lo, hi, new):
        old = self.scales[s][b, h, t]
        scale = scale_of(new, self.fmt)
        if lo:
            scale = np.float32(np.nan) if np.isnan(scale) or np.isnan(old) else max(scale, old)
        at = offsets(s, self.dh)
        out = self.codes[s][b, h, t]
        # the values that the older tokens stood for: fp32 products
        held = (self.block(s, b, h, t)[:lo].astype(np.float32) * old).astype(np.float64) if lo else new[:0]
        with np.errstate(invalid="ignore"):
            if not scale > 0:
                out[at[:hi]] = 0
            else:
                x = np.concatenate([held, new]) / np.float64(scale)
                out[at[:hi]] = to_bytes(nearest(x, self.fmt), self.fmt)
        self.scales[s][b, h, t] = scale

    def values(self, s, b, n):
        """The first n tokens of sequence b, [H, n, dh] float64 (code * scale exactly)."""
        T = (n + BLOCK - 1) // BLOCK
        x = from_bytes(self.codes[s][b, :, :T][..., offsets(s, self.dh)], self.fmt)
        return (x * self.scales[s][b, :, :T, None, None].astype(np.float64)).reshape(self.H, T * BLOCK, self.dh)[:, :n]

    def read(self, first, count, n, dtype):
        out = {}
        for s in "kv":
            o = np.zeros((self.B, n, self.H * self.dh))
            for b in range(self.B):
                f, c = int(first[b]), int(np.clip(count[b], 0, n))
                if f < 0 or f + c > self.cap or c == 0:
                    continue
                x = self.values(s, b, f + c)[:, f:].transpose(1, 0, 2).reshape(c, -1)
                o[b, :c] = round_to(x.astype(np.float32), dtype)       # fp32 product, then the storage type
            out[s] = o
        return out


def attention(cache, q, lengths, waves=4):
    """q [B, n, hq, dh] float64 -> (out, tol): query token i of n sees lengths[b] - (n - 1 - i) tokens.

    tol bounds the fp32 kernel's error per (sequence, query, head).  With S = max_t sum_d |q_d k_td| / sqrt(dh): a
    logit is dh products summed by matrix instructions (up to 8 units of 2^-24 of the block's absolute sum for one,
    measured below 4.6, and one rounding for each of the at most 12 that follow each other), two roundings of the
    factor, one of the difference to the maximum: at most 25 * 2^-24 S.  It changes a weight by that relative
    amount, and the sum by no more: 50 S.  exp2 is within 2^-22, twice: 8.  A lane adds 16 weights a block and a
    matrix instruction chain six roundings a block, over at most t blocks of one wave; weights of 22 bits, scale
    and merges: 32 together.  All relative to sum p |v| / sum p <= max |v|.  `waves` take a pair's blocks in turn."""
    B, n, hq, dh = q.shape
    G = hq // cache.H
    out, tol = np.zeros((B, n, hq, dh)), np.zeros((B, n, hq))
    for b in range(B):
        N = int(lengths[b])
        k, v = (cache.values(s, b, N) for s in "kv")
        for i in range(n):
            m = N - (n - 1 - i)
            if m <= 0:
                continue
            for h in range(hq):
                kk, vv = k[h // G, :m], v[h // G, :m]
                z = kk @ q[b, i, h] / np.sqrt(dh)
                p = np.exp(z - z.max())
                out[b, i, h] = p @ vv / p.sum()
                S = (np.abs(kk) @ np.abs(q[b, i, h])).max() / np.sqrt(dh)
                t = (N + BLOCK - 1) // BLOCK // waves + 1
                tol[b, i, h] = (50 * S + 22 * t + 40) * 2.0 ** -24 * np.abs(vv).max()
    return out, tol


def norm_rope(x, weight, eps, positions, theta):
    """x [T, heads, dh] float64; weight [dh] or None; theta 0: not rotated."""
    dh = x.shape[-1]
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    if theta == 0:
        return x
    # long double: the angle of a far position to 2^-40 of a revolution
    f = np.longdouble(theta) ** (-np.arange(dh // 2, dtype=np.longdouble) * 2 / dh)
    turns = np.asarray(positions, dtype=np.longdouble)[:, None, None] * f / (2 * np.longdouble(np.pi))
    a = ((turns - np.rint(turns)) * 2 * np.longdouble(np.pi)).astype(np.float64)
    lo, hi = x[..., :dh // 2], x[..., dh // 2:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)
