"""Plain reference of packed caches (include/kvr.h), in numpy: rounding, layout and
attention in 64 bits.  Test infrastructure; it shares no code with the library.

A code is the nearest integer to a quotient, so the single fp32 operations that the
format states are carried out as such: one operation on fp32 values in float64,
rounded once to fp32, is that fp32 operation (53 >= 2 * 24 + 2 bits).
"""
from __future__ import annotations

import numpy as np

F32, F64 = np.float32, np.float64


def width(hd: int) -> int:
    return 64 if hd <= 64 else 128


def block_bytes(hd: int, bits: int) -> int:
    return 4 * width(hd) * bits + 32 * (width(hd) // 64) * 4


def blocks(n_cap: int) -> int:
    return (n_cap + 31) // 32


def bf16_down(x: np.ndarray) -> np.ndarray:
    """fp32 to the largest bf16 not above it."""
    u = np.ascontiguousarray(x, F32).view(np.uint32)
    cut = u & np.uint32(0xFFFF0000)
    away = (u >> 31 == 1) & (cut != u)
    return (cut + np.where(away, np.uint32(0x10000), np.uint32(0))).astype(np.uint32).view(F32)


def bf16_up_positive(x: np.ndarray) -> np.ndarray:
    u = np.ascontiguousarray(x, F32).view(np.uint32).astype(np.uint64)
    return ((u + 0xFFFF) & 0xFFFF0000).astype(np.uint32).view(F32)


def quantise(x: np.ndarray, bits: int):
    """x [..., hd] fp32 -> codes [..., hd] int, scale and offset [..., groups] fp32."""
    x = np.asarray(x, F32)
    hd, top = x.shape[-1], (1 << bits) - 1
    groups = width(hd) // 64
    codes = np.zeros(x.shape, np.int64)
    scale = np.zeros((*x.shape[:-1], groups), F32)
    offset = np.zeros((*x.shape[:-1], groups), F32)
    with np.errstate(all="ignore"):
        for g in range(groups):
            y = x[..., 64 * g:64 * g + 64]
            lo, hi = y.min(-1), y.max(-1)
            m = bf16_down(lo)
            t = (hi.astype(F64) - m).astype(F32)
            s = bf16_up_positive((t.astype(F64) * F32(1.0 / top)).astype(F32))
            s = np.where(t > 0, np.maximum(s, F32(2.0 ** -126)), F32(0))
            good = np.isfinite(y).all(-1) & np.isfinite(t) & np.isfinite(s)
            s, m = np.where(good, s, F32(0)), np.where(good, m, F32(np.nan))
            inv = np.where(s > 0, (1.0 / s.astype(F64)).astype(F32), F32(0))
            d = (y.astype(F64) - m[..., None]).astype(F32)
            c = np.rint((d.astype(F64) * inv[..., None]).astype(F32))
            codes[..., 64 * g:64 * g + 64] = np.where(good[..., None], np.clip(np.nan_to_num(c), 0, top), 0).astype(np.int64)
            scale[..., g], offset[..., g] = s, m
    return codes, scale, offset


def values(codes, scale, offset) -> np.ndarray:
    """What they stand for, float64 [..., hd]."""
    g = np.arange(codes.shape[-1]) // 64
    with np.errstate(all="ignore"):
        return offset[..., g].astype(F64) + scale[..., g].astype(F64) * codes


def code_place(hd: int, bits: int, value: bool, r: int, d: int):
    """(byte of the block, bit it starts at) of position r, dimension d."""
    w = width(hd)
    if value:
        lane = (r // 4 % 4) * 16 + d % 16
        if bits == 4:
            return ((lane * (w // 32) + d // 32) * 2 + r // 16) * 4 + r % 4, 4 * (d // 16 % 2)
        return ((lane * (w // 16) + d // 16) * 2 + r // 16) * 4 + r % 4, 0
    q = ((r // 16 * 4 + d // 8 % 4) * 16 + r % 16) * (w // 32) + d // 32
    if bits == 4:
        nib = (d % 2) * 4 + d % 8 // 2
        return q * 4 + nib // 2, 4 * (nib % 2)
    return q * 8 + d % 8, 0


def _places(hd, bits, value):
    at = [[code_place(hd, bits, value, r, d) for d in range(hd)] for r in range(32)]
    a = np.array(at)
    return a[..., 0], a[..., 1]


def write(packed: np.ndarray, rows: np.ndarray, positions, bits: int, value: bool) -> None:
    """Quantise rows [H, len(positions), hd] into planes packed [H, blocks, bytes] (uint8), in place."""
    hd = rows.shape[-1]
    w = width(hd)
    byte, bit = _places(w, bits, value)
    codes, scale, offset = quantise(rows, bits)
    codes = np.concatenate([codes, np.zeros((*codes.shape[:-1], w - hd), np.int64)], -1)  # dimensions behind head_dim
    groups, cb = scale.shape[-1], 4 * width(hd) * bits
    word = (offset.view(np.uint32) & np.uint32(0xFFFF0000)) | (scale.view(np.uint32) >> np.uint32(16))
    nan = np.isnan(offset)
    word = np.where(nan, np.uint32(0x7FC00000), word).astype("<u4")
    mask = (1 << bits) - 1
    for i, p in enumerate(positions):
        b, r = p // 32, p % 32
        for d in range(w):
            at, sh = byte[r, d], bit[r, d]
            packed[:, b, at] = (packed[:, b, at] & (0xFF ^ (mask << sh))) | (codes[:, i, d] << sh).astype(np.uint8)
        at = cb + r * groups * 4
        packed[:, b, at:at + 4 * groups] = np.ascontiguousarray(word[:, i]).view(np.uint8).reshape(packed.shape[0], -1)


def read(packed: np.ndarray, n: int, hd: int, bits: int, value: bool):
    """Planes [H, blocks, bytes] -> (codes [H, n, hd], scale, offset [H, n, groups])."""
    byte, bit = _places(hd, bits, value)
    p = np.arange(n)
    b, r = p // 32, p % 32
    codes = (packed[:, b[:, None], byte[r]] >> bit[r].astype(np.uint8)) & ((1 << bits) - 1)
    groups, cb = width(hd) // 64, 4 * width(hd) * bits
    at = cb + (r[:, None] * groups + np.arange(groups)[None, :]) * 4
    raw = sum(packed[:, b[:, None], at + k].astype(np.uint32) << np.uint32(8 * k) for k in range(4)).astype(np.uint32)
    return codes.astype(np.int64), (raw << np.uint32(16)).view(F32), (raw & np.uint32(0xFFFF0000)).view(F32)


def attend(q: np.ndarray, positions, k: np.ndarray, v: np.ndarray) -> np.ndarray:
    """q [R, Hq, hd]; k, v [Hkv, n, hd] float64.  Row r sees slots 0 .. positions[r]; none: zeros."""
    R, Hq, hd = q.shape
    G = Hq // k.shape[0]
    out = np.zeros((R, Hq, hd), F64)
    with np.errstate(all="ignore"):
        for r in range(R):
            n = int(positions[r]) + 1
            if n <= 0:
                continue
            for g in range(k.shape[0]):
                s = q[r, g * G:(g + 1) * G].astype(F64) @ k[g, :n].T / np.sqrt(hd)
                w = np.exp(s - s.max(1, keepdims=True))
                out[r, g * G:(g + 1) * G] = (w / w.sum(1, keepdims=True)) @ v[g, :n]
    return out


def attend_bound(q, positions, kc, vc, bits: int, fp32: bool, pairs: bool = False) -> np.ndarray:
    """Bound on |kernel - attend| per row and head [R, Hq], without the output's own rounding; kc, vc: (codes, scale,
    offset) of the keys and values.

    u = 2^-24.  The matrix operands are b = 16 + code < 32 (4 bits) or the code < 256, so a product's terms are at
    most |q| (b s + |m|) =: |q| K with K the largest over the row's keys, and the values' at most b s + |m| =: V.
      score: hd products and a few sums, each off by u of a partial sum of at most A = sum_d |q_d| K / sqrt(hd):
        dS <= (hd + 16) u A, plus 4 u |S| <= 4 u A from the scaling into the exponent and 2^-22 for the exponential
      probability: off by dS + 2^-22 relative; numerator and denominator both: twice that times V
      p s as bf16 pieces: 2 pieces 2^-16, 3 pieces 2^-24 of a term, relative: times V
      the sums over n keys: at most n / 32 + 64 additions in a row, u of a partial sum each: times V, for both
    pairs: the kernel for many rows holds keys, values and probabilities as sums of two bf16, each off by 2^-16 relative
      (half a step of the second piece, 2^-8 of at most 2^-8), and leaves out the product of the two second pieces of
      values and probabilities, 2^-16: dS <= 2^-16 A more, outputs 2 * 2^-16 V more."""
    u = 2.0 ** -24
    big = 32.0 if bits == 4 else 256.0
    R, Hq, hd = q.shape
    Hkv = kc[0].shape[0]
    G = Hq // Hkv
    out = np.zeros((R, Hq))
    for r in range(R):
        n = int(positions[r]) + 1
        if n <= 0:
            continue
        for h in range(Hq):
            g = h // G
            K = float((big * kc[1][g, :n].astype(F64) + np.abs(kc[2][g, :n].astype(F64))).max())
            V = float((big * vc[1][g, :n].astype(F64) + np.abs(vc[2][g, :n].astype(F64))).max())
            A = float(np.abs(q[r, h].astype(F64)).sum()) * K / np.sqrt(hd)
            dS = ((hd + 20) * u + (2.0 ** -16 if pairs else 0.0)) * A + 2.0 ** -22
            out[r, h] = V * (2 * (dS + 2.0 ** -22) + (u if fp32 else 2.0 ** -16) +
                             (2.0 ** -15 if pairs else 0.0) + 2 * (n / 32 + 64) * u)
    return out
