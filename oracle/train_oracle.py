"""CPU oracle of microscaled 4-bit floating point and of distillation from a teacher's top logits: plain double-precision numpy
from the definitions, sharing no code with the CUDA path.  TEST INFRASTRUCTURE ONLY.

* ``mx_quantize`` / ``mx_codes`` / ``mx_values``  the OCP "MXFP4" format: blocks of 32, power-of-two scales (byte 255: NaN),
  elements of sign, two exponent bits and one mantissa bit.
* ``mx_linear``  the product of two microscaled matrices, with the sum of the products' magnitudes for error bounds.
* ``distill``    loss and gradient, token by token, entry by entry.
"""
from __future__ import annotations

import numpy as np

ELEMENTS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])



def mx_quantize(x, inv_smooth=None):
    """x [M, K] of any float type -> (element codes uint8 [M, 32 * blocks], scale bytes uint8 [M, blocks])."""
    x = np.asarray(x, dtype=np.float64)
    if inv_smooth is not None:
        with np.errstate(over="ignore", invalid="ignore"):
            x = (x * np.asarray(inv_smooth, dtype=np.float64)).astype(np.float32).astype(np.float64)
    M, K = x.shape
    blocks = -(-K // 32)
    t = np.zeros((M, blocks * 32))
    t[:, :K] = x
    codes, scales = np.zeros((M, blocks * 32), dtype=np.uint8), np.zeros((M, blocks), dtype=np.uint8)
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    for b in range(blocks):
        block = t[:, 32 * b:32 * b + 32]
        top = np.abs(block).max(axis=1)
        fine = np.isfinite(top)
        _, e = np.frexp(np.where(fine, top, 0.0))            # top = f * 2^e, f in [1/2, 1)
        e = np.where(top == 0, 0, np.maximum(e - 1 - 2, -127))
        scales[:, b] = np.where(fine, e + 127, 255)
        a = np.ldexp(np.abs(np.where(fine[:, None], block, 0.0)), -e[:, None])
        below = np.searchsorted(borders, a, side="left")     # borders less than a; a border itself belongs to the even neighbour
        above = np.searchsorted(borders, a, side="right")
        index = np.where(above % 2 == 0, above, below)
        sign = np.signbit(np.where(fine[:, None], block, 0.0))
        codes[:, 32 * b:32 * b + 32] = index + 8 * sign
    return codes, scales


def mx_codes(codes):
    """Element codes -> packed bytes, the even column in the low nibble."""
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def mx_values(packed, scales, K=None):
    """What packed codes and scale bytes stand for, float64 [M, K]."""
    packed, scales = np.asarray(packed), np.asarray(scales)
    codes = np.empty((packed.shape[0], packed.shape[1] * 2), dtype=np.uint8)
    codes[:, 0::2], codes[:, 1::2] = packed & 15, packed >> 4
    v = ELEMENTS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    v = v * np.repeat(s, 32, axis=1)
    return v if K is None else v[:, :K]


def mx_linear(w_packed, w_scales, x_packed, x_scales):
    """(y float64 [M, N], sum of the products' magnitudes [M, N])."""
    w, x = mx_values(w_packed, w_scales), mx_values(x_packed, x_scales)
    return x @ w.T, np.abs(x) @ np.abs(w).T


def distill(z, idx, top, tau=1.0, teacher_lse=None, weight=None):
    """z [T, V], idx [T, k], top [T, k] -> (loss [T], gradient [T, V], stats [T, 2], the terms' magnitudes for error bounds: of the
    loss [T], of the gradient [T, V])."""
    z, top = np.asarray(z, dtype=np.float64), np.asarray(top, dtype=np.float64)
    T, V = z.shape
    loss, grad, stats = np.zeros(T), np.zeros((T, V)), np.full((T, 2), np.nan)
    loss_size, grad_size = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        w = 1.0 if weight is None else float(weight[t])
        if w == 0.0:
            continue
        m = z[t].max()
        e = np.exp((z[t] - m) / tau)
        s = e.sum()
        stats[t] = m, s
        q, logq = e / s, (z[t] - m) / tau - np.log(s)
        entries = [j for j in range(idx.shape[1]) if 0 <= idx[t, j] < V and top[t, j] > -np.inf]
        if not entries:
            continue
        a = top[t, entries] / tau
        norm = a.max() + np.log(np.exp(a - a.max()).sum()) if teacher_lse is None else float(teacher_lse[t])
        p = np.exp(a - norm)
        at = idx[t, entries].astype(np.int64)
        with np.errstate(invalid="ignore"):
            terms = np.where(p != 0, p * ((a - norm) - logq[at]), 0.0)       # p = 0 adds nothing, whatever q is
        loss[t], loss_size[t] = w * terms.sum(), abs(w) * (np.abs(terms) + p).sum()
        grad[t] = p.sum() * q
        grad_size[t] = p.sum() * q
        for v, pv in zip(at, p):
            grad[t, v] -= pv
            grad_size[t, v] += pv
        grad[t] *= w / tau
        grad_size[t] *= abs(w) / tau
    return loss, grad, stats, loss_size, grad_size
