"""The dense product, dropout and the balance loss in float64 numpy, straight from their definitions in switch_moe.h, and the
bounds that the kernels' arithmetic implies."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2101_03961_b200 import switch_moe as sm

HALF_STEP = {sm.BF16: 2.0**-8, sm.F32: 2.0**-24}              # torch.finfo(t).eps / 2: one rounding, relative
TYPES = {sm.BF16: torch.bfloat16, sm.F32: torch.float32}


def philox4x32_10(counter, key):
    """uint32 [n, 4] of counters [n, 4] (Salmon et al., 2011)."""
    c = [np.ascontiguousarray(counter[:, i]).astype(np.uint64) for i in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, axis=1).astype(np.uint32)


def dropout_factors(rows, cols, rate, site, key, offset, row0=0):
    """Float64 [rows, cols]: 0 or 65536 / (65536 - q), for the rows from row0 on."""
    q = int(math.floor(rate * 65536 + 0.5))
    if q == 0:
        return np.ones((rows, cols))
    per_row = (cols + 7) // 8
    b = row0 * per_row + np.arange(rows * per_row, dtype=np.uint64)
    counter = np.zeros((b.size, 4), dtype=np.uint64)
    counter[:, 0] = b & np.uint64(0xFFFFFFFF)
    counter[:, 1] = (b >> np.uint64(32)) + np.uint64(site << 16)
    counter[:, 2], counter[:, 3] = offset & 0xFFFFFFFF, offset >> 32
    words = philox4x32_10(counter, (key & 0xFFFFFFFF, key >> 32))
    halves = np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(rows, per_row * 8)[:, :cols]
    return np.where(halves >= q, 65536.0 / (65536 - q), 0.0)


_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, kind):
    if kind == sm.ACT_RELU:
        return np.where(z < 0, 0.0, z)
    return z * 0.5 * (1 + _erf(z / math.sqrt(2))) if kind == sm.ACT_GELU else z


def d_act(z, kind):
    if kind == sm.ACT_RELU:
        return (z > 0).astype(np.float64)
    if kind == sm.ACT_GELU:
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


# What a product of contraction length K may be off, in units of sum |a b|.  bf16: the tensor pipe truncates; per step of 16
# products up to 17 addends are cut below 2^-23 of the largest and the running sum is cut once, and (a contraction cut into
# parts) 16 parts are added with one rounding each.  Float32: six of nine part products (2^-25), the same cuts inside an
# accumulator's life of 64 steps at the size of that block's sum, then one rounding per block, and two scalings by powers of 2.
def product_error(dtype, K):
    if dtype == sm.BF16:
        return (17 + K / 16 + 1) * 2.0**-23 + 16 * 2.0**-24
    return 2.0**-25 + (17 + 4 + 1) * 2.0**-23 + (K / 64 + 1) * 2.0**-24 + 16 * 2.0**-24


# Phi and GELU' from Abramowitz and Stegun 7.1.26: 1.5e-7 for erf, float32 arithmetic around it
GELU_ERROR = 5e-7


def rows_tensor(a, dtype, pad, fill=float("nan")):
    """numpy [rows, cols] -> device tensor whose rows are padded by `pad` elements (on top of 16 bytes) that hold `fill`."""
    unit = 8 if dtype == sm.BF16 else 4
    rows, cols = a.shape
    ld = (cols + unit - 1) // unit * unit + pad
    t = torch.full((max(rows, 1), ld), fill, dtype=TYPES[dtype], device="cuda")
    t[:rows, :cols] = torch.from_numpy(a).to(TYPES[dtype])
    return t[:rows, :cols], t


def to64(t):
    return t.detach().double().cpu().numpy()


def balance(logits, index, mask, k, groups, alpha, d_loss):
    """loss, counts, tokens, dlogits from float64 logits [T, E]."""
    T, E = logits.shape
    per = T // groups
    loss, counts, tokens, grad = 0.0, np.zeros((groups, E), np.int64), np.zeros(groups, np.int64), np.zeros((T, E))
    for g in range(groups):
        rows = np.arange(g * per, (g + 1) * per)
        use = [t for t in rows if (mask is None or mask[t]) and not np.all(np.isneginf(logits[t]))]
        p = {}
        for t in use:
            e = np.exp(logits[t] - np.nanmax(logits[t])) if not np.all(np.isnan(logits[t])) else logits[t]
            p[t] = e / e.sum()
            if index is None:
                left = np.where(np.isnan(logits[t]), -np.inf, logits[t])
                for _ in range(k):
                    best = int(np.argmax(left))
                    if np.isneginf(left[best]):
                        break
                    counts[g, best] += 1
                    left[best] = -np.inf
            else:
                for e in index[t]:
                    if 0 <= e < E:
                        counts[g, e] += 1
        n = tokens[g] = len(use)
        if n == 0:
            continue
        f = counts[g] / (k * n)
        loss += alpha * E * float((f * sum(p.values())).sum()) / n / groups
        up = d_loss * alpha * E / groups / n * f
        for t in use:
            grad[t] = p[t] * (up - (p[t] * up).sum())
    return loss, counts, tokens, grad
