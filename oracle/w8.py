"""The 8-bit linear: quantizers, exact sums and the epilogue, stated plainly on the CPU (test infrastructure).

The readings of the 4-bit quantizers (:mod:`oracle.quant`) with 127 in place of 7: rounding half to even, the symmetric
range, an exact rational clip ratio, one scale per token and per output channel (Eq. (1), Sec. 4.1).
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

from . import hadamard, quant

LARGEST = 127


def codes(X: np.ndarray, clip=(1, 1)) -> np.ndarray:
    """sign(X) min(127, rne(127 den |X| / (num A))), A = max |X| of each row, decided on the fp64 values as rationals.

    The fp64 quotient is off by at most a few 2^-53 of its value (below 2^12), so away from a half it rounds as the exact one; near
    one (1e-9) the rationals decide."""
    num, den = int(clip[0]), int(clip[1])
    X = np.asarray(X, dtype=np.float64)
    A = np.abs(X).max(axis=1, keepdims=True)
    v = np.where(A > 0, np.abs(X) * (LARGEST * den) / np.where(A > 0, A * num, 1.0), 0.0)
    q = np.minimum(quant.rne(v), LARGEST)
    for m, k in zip(*np.nonzero(np.abs(np.abs(v - np.floor(v)) - 0.5) < 1e-9)):
        r = LARGEST * den * abs(Fraction(float(X[m, k]))) / (num * Fraction(float(A[m, 0])))
        f = r.numerator // r.denominator
        up = r - f > Fraction(1, 2) or (r - f == Fraction(1, 2) and f % 2 == 1)
        q[m, k] = min(f + up, LARGEST)
    return (np.sign(X) * q).astype(np.int8)


def act_quant8(x: np.ndarray, b: int, clip=(1, 1)):
    """Rotate and quantize tokens [M, K] (fp16, or fp32 arrays of bf16 values): (q int8 [M, K], s_x fp32 [M])."""
    num, den = int(clip[0]), int(clip[1])
    if x.dtype == np.float16:
        X = hadamard.rotate_act_units(x, b).astype(np.float64) * 2.0 ** -24   # integers below 2^53: exact
    else:
        X = hadamard.rotate_act_staged(x, b)
    A = np.abs(X).max(axis=1)
    s_x = (A * float(num)) / ((float(den) * float(LARGEST)) * float(np.sqrt(np.float64(b))))
    return codes(X, clip), s_x.astype(np.float32)


def quantize_weights8(W_rot: np.ndarray):
    """s_w = fp16(max|row| / 127), q = clip(rne(w / s_w), -127, 127) against the stored scale; zeros where that is 0."""
    W = np.asarray(W_rot, dtype=np.float64)
    s_w = quant.fp16_scale(np.abs(W).max(axis=1) / float(LARGEST))
    s = s_w.astype(np.float64)
    q = np.zeros(W.shape, dtype=np.int8)
    nz = s > 0
    q[nz] = np.clip(quant.rne(W[nz] / s[nz, None]), -LARGEST, LARGEST).astype(np.int8)
    return q, s_w


def epilogue(acc: np.ndarray, s_x: np.ndarray, s_w: np.ndarray) -> np.ndarray:
    """fp32(fp32(acc) s_x) s_w, each product rounded to fp32: the value that is rounded once to the outputs' type."""
    t = np.asarray(acc).astype(np.float32) * np.asarray(s_x, np.float32)[:, None]
    return t * np.asarray(s_w, np.float16).astype(np.float32)[None, :]
