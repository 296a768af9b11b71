"""CPU oracle of the few-token operators: weights in 4 bits, the routed projection over a few tokens, the FFN-MoE layer on
a routing decision that may name an expert twice or one that does not exist.  numpy, 64 bits, written from the
definitions in include/rom.h; each product also comes with the sum of its terms' sizes, which is what rounding errors of
a sum are measured against."""
from __future__ import annotations

import numpy as np

F64 = np.float64
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def to_bf16(v):
    """Nearest bf16 (ties to even) of float32 values, as float64; NaN stays NaN."""
    f = np.asarray(v, np.float32)
    bits = f.view(np.uint32).astype(np.uint64)
    out = ((bits + 0x7FFF + ((bits >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(f), np.float32(np.nan), out).astype(F64)


def q4_quantize(w, group):
    """w [E, rows, cols] -> (codes uint8 [E, rows, cols], scales float64 [E, rows, groups])."""
    w = np.asarray(w, np.float32)
    E, rows, cols = w.shape
    n = -(-cols // group)
    padded = np.zeros((E, rows, n * group), np.float32)
    padded[:, :, :cols] = w
    v = padded.reshape(E, rows, n, group)
    with np.errstate(invalid="ignore", over="ignore"):
        scales = to_bf16((np.abs(v).max(-1).astype(F64) / 6.0).astype(np.float32))
    bad = ~np.isfinite(v).all(-1)
    scales[bad] = np.nan
    codes = np.zeros(v.shape, np.uint8)
    for e, r, g in np.argwhere(~bad & (scales > 0)):
        a = np.abs(v[e, r, g].astype(F64)) / scales[e, r, g]       # bf16 / bf16 or fp32 / bf16 in 64 bits
        low = np.clip(np.searchsorted(E2M1, a, side="right") - 1, 0, 6)
        mid = (E2M1[low] + E2M1[low + 1]) / 2
        up = (np.abs(v[e, r, g].astype(F64)) > mid * scales[e, r, g]) | ((np.abs(v[e, r, g].astype(F64)) == mid * scales[e, r, g]) & (low % 2 == 1))
        m = low + up
        codes[e, r, g] = np.where(m > 0, m + 8 * (v[e, r, g] < 0), 0)
    return codes.reshape(E, rows, -1)[:, :, :cols], scales


def q4_values(codes, scales, group):
    E, rows, cols = codes.shape
    s = np.repeat(scales, group, axis=2)[:, :, :cols]
    return np.where(codes >= 8, -1.0, 1.0) * E2M1[codes & 7] * s


def q4_layout(codes, scales, group):
    """The packed bytes, one weight at a time."""
    E, rows, cols = codes.shape
    rp, cp = -(-rows // 16) * 16, -(-cols // 128) * 128
    out = np.zeros(E * rp * cp // 2, np.uint8)
    e, r, k = np.meshgrid(np.arange(E), np.arange(rows), np.arange(cols), indexing="ij")
    block = (e * (rp // 16) + r // 16) * (cp // 128) + k // 128
    at = block * 1024 + ((k % 32) // 8 * 16 + r % 16) * 16 + (k % 128) // 32 * 4 + (k % 8) // 2
    np.add.at(out, at.ravel(), (codes.astype(np.uint16) << (4 * (k % 2))).astype(np.uint8).ravel())
    s = np.zeros(E * rp * (cp // group), np.uint16)
    e, r, g = np.meshgrid(np.arange(E), np.arange(rows), np.arange(scales.shape[2]), indexing="ij")
    bits = (scales.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    s[((e * (rp // 16) + r // 16) * (cp // group) + g) * 16 + r % 16] = np.where(np.isnan(scales), 0x7FC0, bits)
    return np.concatenate([out, s.view(np.uint8)])


def project(x, w, idx, gate=None, row_scale=None, residual=None):
    """(out [N, rows], size of the terms [N, rows]); x [N, cols] or [N, K, cols]; idx [N, K]."""
    x, w = np.asarray(x, F64), np.asarray(w, F64)
    N, K = idx.shape
    w_size = np.abs(w)
    out, size = np.zeros((N, w.shape[1])), np.zeros((N, w.shape[1]))
    for n in range(N):
        for k in range(K):
            e = idx[n, k]
            if e < 0 or e >= w.shape[0]:
                continue
            v = x[n, k] if x.ndim == 3 else x[n]
            g = 1.0 if gate is None else float(gate[n, k])
            out[n] += g * (w[e] @ v)
            size[n] += abs(g) * (w_size[e] @ np.abs(v))
    if row_scale is not None:
        out, size = out * np.asarray(row_scale, F64)[:, None], size * np.abs(np.asarray(row_scale, F64))[:, None]
    return (out if residual is None else out + np.asarray(residual, F64)), size


def ffn_step(x, w_gate_up, w_down, idx, gate, pre_norm, eps, skip):
    """(out [N, D], size of the terms of out, relative error of SiLU(gate) * up per unit of summation error, as a size).

    w_gate_up [E, 2 d_ff, D]: gate rows, then up rows.  The second size is sum_f |w_down| * d h, d h the change of
    h = SiLU(a) b for changes of a and b by the sizes of their own terms (|SiLU'| <= 1.1)."""
    x, wg, wd = np.asarray(x, F64), np.asarray(w_gate_up, F64), np.asarray(w_down, F64)
    N, K = idx.shape
    f = wg.shape[1] // 2
    wg_size, wd_size = np.abs(wg), np.abs(wd)
    xn = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) if pre_norm else x
    out, size, carried = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    for n in range(N):
        for k in range(K):
            e = idx[n, k]
            if e < 0 or e >= wg.shape[0]:
                continue
            a, b = wg[e, :f] @ xn[n], wg[e, f:] @ xn[n]
            sa, sb = wg_size[e, :f] @ np.abs(xn[n]), wg_size[e, f:] @ np.abs(xn[n])
            s = a / (1.0 + np.exp(-a))
            g = float(gate[n, k])
            out[n] += g * (wd[e] @ (s * b))
            size[n] += abs(g) * (wd_size[e] @ np.abs(s * b))
            carried[n] += abs(g) * (wd_size[e] @ (1.1 * sa * np.abs(b) + np.abs(s) * sb + np.abs(s * b) * (np.abs(a) + 4)))
    return (out + x if skip else out), size, carried
