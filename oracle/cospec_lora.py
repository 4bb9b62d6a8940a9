"""Low-rank adapters in float64 -- TEST INFRASTRUCTURE ONLY, written from the definitions: for a row m with adapter a
  y = x W^T + c_a drop(x) A_a^T B_a^T,  c_a = scaling_a / (1 - p),
the dropout mask a function of the element's place through Philox4x32-10, and the gradients for x, A and B."""
from __future__ import annotations

import numpy as np

from oracle.philox import philox4x32_10


def keep_mask(rows: int, width: int, dropout: float, seed: int, site: int):
    """(mask [rows, width] of 0 and 1, share kept): column k of row m stays where the 16 bits number k mod 8 of the draw
    at counter (k // 8, m, site, 2) are at least round(65536 dropout)."""
    thr = int(np.floor(float(np.float32(dropout)) * 65536 + 0.5))
    mask = np.ones((rows, width))
    if thr:
        oct_ = np.arange((width + 7) // 8, dtype=np.uint64)
        for m in range(rows):
            words = philox4x32_10(oct_, np.full(oct_.shape, m), np.full(oct_.shape, site), np.full(oct_.shape, 2), seed & 0xFFFFFFFF, seed >> 32)
            for k in range(width):
                bits = (int(words[(k % 8) // 2][k // 8]) >> (16 * (k % 2))) & 0xFFFF
                mask[m, k] = bits >= thr
    return mask, (65536 - thr) / 65536.0


def forward(x, w, a, b, scaling, adapter, mask=None, kept=1.0):
    """(y, u), and the sums of absolute products behind them for the tests' error bounds."""
    mask = np.ones(x.shape) if mask is None else mask
    y, ay = x @ w.T, np.abs(x) @ np.abs(w).T
    u, au = np.zeros((len(x), a.shape[1])), np.zeros((len(x), a.shape[1]))
    alow = np.zeros(y.shape)
    for m, i in enumerate(adapter):
        if i < 0:
            continue
        c, xm = scaling[i] / kept, np.where(mask[m] > 0, x[m], 0.0)
        u[m], au[m] = c * (a[i] @ xm), abs(c) * (np.abs(a[i]) @ np.abs(xm))
        y[m] += b[i] @ u[m]
        alow[m] = np.abs(b[i]) @ np.abs(u[m])
    return dict(y=y, u=u, abs_y=ay, abs_u=au, abs_low=alow)


def backward(dy, x, w, a, b, scaling, adapter, u, mask=None, kept=1.0):
    mask = np.ones(x.shape) if mask is None else mask
    dx, adx = dy @ w, np.abs(dy) @ np.abs(w)
    t, at = np.zeros((len(x), a.shape[1])), np.zeros((len(x), a.shape[1]))
    da, db, ada, adb = np.zeros(a.shape), np.zeros(b.shape), np.zeros(a.shape), np.zeros(b.shape)
    alow = np.zeros(dx.shape)
    for m, i in enumerate(adapter):
        if i < 0:
            continue
        c, xm = scaling[i] / kept, np.where(mask[m] > 0, x[m], 0.0)
        t[m], at[m] = c * (dy[m] @ b[i]), abs(c) * (np.abs(dy[m]) @ np.abs(b[i]))
        dx[m] += np.where(mask[m] > 0, t[m] @ a[i], 0.0)
        alow[m] = np.abs(t[m]) @ np.abs(a[i])
        da[i] += np.outer(t[m], xm)
        db[i] += np.outer(dy[m], u[m])
        ada[i] += np.outer(at[m], np.abs(xm))
        adb[i] += np.abs(np.outer(dy[m], u[m]))
    return dict(dx=dx, da=da, db=db, t=t, abs_dx=adx, abs_low=alow, abs_da=ada, abs_db=adb, abs_t=at)
