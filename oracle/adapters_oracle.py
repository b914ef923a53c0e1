"""CPU oracle of the low-rank adapters and the counter-based dropout, in 64 bits, written from their definitions.

    out_t = base_t + s_a B_a A_a xd_t,  xd = x or its dropout,  a = row_adapter[t] (outside [0, n): out_t = base_t)
    keep(t, 8 c + j): 16-bit half j of Philox 4x32-10 on (c, t, offset low, offset high) under (seed low, seed high) >= thr

Test infrastructure only.
"""
from __future__ import annotations

import numpy as np

MULT = (0xD2511F53, 0xCD9E8D57)          # Philox 4x32 (Salmon, Moraes, Dror, Shaw, SC 2011)
WEYL = (0x9E3779B9, 0xBB67AE85)


def philox(counter, key, rounds: int = 10) -> np.ndarray:
    """The four output words for counters [..., 4] and a key (2 words), all uint32."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(rounds):
        p = [np.uint64(MULT[0]) * c[0], np.uint64(MULT[1]) * c[2]]
        hi = [v >> np.uint64(32) for v in p]
        lo = [v & np.uint64(0xFFFFFFFF) for v in p]
        c = [hi[1] ^ c[1] ^ np.uint64(k[0]), lo[1], hi[0] ^ c[3] ^ np.uint64(k[1]), lo[0]]
        k = [(k[0] + WEYL[0]) % 2**32, (k[1] + WEYL[1]) % 2**32]
    return np.stack(c, axis=-1).astype(np.uint32)


def threshold(p: float) -> int:
    return int(np.floor(p * 65536 + 0.5))


def keep_mask(rows: int, cols: int, p: float, seed: int, offset: int = 0, row0: int = 0) -> np.ndarray:
    blocks = -(-cols // 8)
    c = np.zeros((rows, blocks, 4), dtype=np.uint32)
    c[..., 0] = np.arange(blocks, dtype=np.uint32)[None, :]
    c[..., 1] = (row0 + np.arange(rows, dtype=np.int64)).astype(np.uint32)[:, None]
    c[..., 2], c[..., 3] = offset % 2**32, offset >> 32
    words = philox(c, (seed % 2**32, seed >> 32))
    draws = np.stack([words & 0xFFFF, words >> 16], axis=-1).reshape(rows, blocks * 8)
    return draws[:, :cols] >= threshold(p)


def dropout(x, p, seed, offset=0, row0=0, residual=None):
    """[rows, cols] in 64 bits; p as held (a multiple of 1 / 65536)."""
    keep = keep_mask(*x.shape, p, seed, offset, row0)
    out = np.where(keep, x.astype(np.float64), 0.0) * (65536.0 / (65536 - threshold(p)))
    return out if residual is None else out + residual.astype(np.float64)


def adapter_forward(x, a, b, ids, scale, base=None):
    """(out, z): x [T, d_in] (a dropout already applied), a [n, r, d_in], b [n, d_out, r], ids [T], scale [n]."""
    n = a.shape[0]
    out = np.zeros((len(x), b.shape[1])) if base is None else base.astype(np.float64).copy()
    z = np.zeros((len(x), a.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < n:
            z[t] = a[i].astype(np.float64) @ x[t]
            out[t] += float(scale[i]) * (b[i].astype(np.float64) @ z[t])
    return out, z


def adapter_backward(dy, x, z, a, b, ids, scale, mask=None, dx_base=None):
    """(dx, grad_a, grad_b); x with its dropout applied, mask: keep * its scale (None: ones)."""
    n = a.shape[0]
    dx = np.zeros(x.shape) if dx_base is None else dx_base.astype(np.float64).copy()
    ga, gb = np.zeros(a.shape), np.zeros(b.shape)
    for t, i in enumerate(ids):
        if 0 <= i < n:
            e = float(scale[i]) * (b[i].astype(np.float64).T @ dy[t])
            g = a[i].astype(np.float64).T @ e
            dx[t] += g if mask is None else g * mask[t]
            ga[i] += np.outer(e, x[t])
            gb[i] += float(scale[i]) * np.outer(dy[t], z[t])
    return dx, ga, gb
