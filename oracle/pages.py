"""The paged KV4 cache: what its kernels compute, stated plainly on the CPU (test infrastructure).

A cache is a pool of pages, rows [pages, Hkv, page] of codes, scales and zero-points as ``oracle.kv4`` defines
them; slot p * page + i is token i of page p.  Quantization decides in fp32 in the written order (``kv4_quant``
for fp16 values; here for any fp32 values, bf16 ones among them); attention is in fp64 on the fp32
reconstructions.
"""
from __future__ import annotations

import numpy as np

from . import kv4, quant


def quantize(x: np.ndarray):
    """(codes 0..15, s fp32, z) of vectors x [..., 128] of fp32 values: the steps of ``kv4.kv4_quant``."""
    f32 = np.float32
    x = np.asarray(x, dtype=f32)
    x_max = np.maximum(x.max(axis=-1), f32(0.0)) * kv4.CLIP
    x_min = np.minimum(x.min(axis=-1), f32(0.0)) * kv4.CLIP
    s = (x_max - x_min) / f32(kv4.LEVELS)
    s = np.where(s == 0.0, f32(1.0), s).astype(f32)
    z = np.clip(quant.rne(-x_min / s), 0, kv4.LEVELS)
    q = np.clip(quant.rne(x / s[..., None]) + z[..., None], 0, kv4.LEVELS)
    return q.astype(np.uint8), s, z.astype(np.uint8)


def append(codes, scales, zeros, x, slots):
    """Write fp32 values x [n, Hkv, 128] into copies of one side of a cache (unpacked codes [pages, Hkv, page, 128]).
    Returns (codes, scales, zeros, values fp32 [n, Hkv, 128]); slots that are no slots are left out."""
    codes, scales, zeros = codes.copy(), scales.copy(), zeros.copy()
    pages, _, page = scales.shape
    q, s, z = quantize(x)
    values = kv4.kv4_dequant(q, s, z)
    for t, slot in enumerate(slots):
        if 0 <= slot < pages * page:
            p, i = divmod(int(slot), page)
            codes[p, :, i], scales[p, :, i], zeros[p, :, i] = q[t], s[t], z[t]
        else:
            values[t] = 0
    return codes, scales, zeros, values


def read(codes, scales, zeros, slots):
    """fp32 values [n, Hkv, 128] of the slots; 0 for one that is none."""
    pages, Hkv, page = scales.shape
    out = np.zeros((len(slots), Hkv, 128), dtype=np.float32)
    for t, slot in enumerate(slots):
        if 0 <= slot < pages * page:
            p, i = divmod(int(slot), page)
            out[t] = kv4.kv4_dequant(codes[p, :, i], scales[p, :, i], zeros[p, :, i])
    return out


def attention(q, k, v, seen):
    """softmax over the seen tokens of q . k / sqrt(d), applied to v, in fp64; rows that see nothing give 0.
    q [n, Hq, d]; k, v [T, Hkv, d] (fp32 reconstructions); seen bool [n, T]."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    n, Hq, d = q.shape
    G = Hq // k.shape[1]
    out = np.zeros((n, Hq, d))
    for i in range(n):
        t = np.flatnonzero(seen[i])
        if len(t) == 0:
            continue
        for h in range(Hq):
            score = k[t, h // G] @ q[i, h] / np.sqrt(float(d))
            p = np.exp(score - score.max())
            out[i, h] = (p / p.sum()) @ v[t, h // G]
    return out


def chain(n, T):
    """Who sees what without a mask: node i of n, the last of T tokens, everything up to itself."""
    return np.arange(T)[None, :] <= (T - n + np.arange(n))[:, None]


def tree(mask, T):
    """With a mask bool [n, n]: all tokens before the nodes, and the nodes it names."""
    n = len(mask)
    return np.concatenate([np.ones((n, max(0, T - n)), dtype=bool), mask[:, :T]], axis=1)


def pack_mask(mask, max_nodes):
    """The words of a mask bool [n, <= max_nodes]: bit j mod 64 of word j / 64, as int64."""
    bits = np.zeros((len(mask), -(-max_nodes // 64) * 64), dtype=bool)
    bits[:, :mask.shape[1]] = mask
    words = np.packbits(bits, axis=1, bitorder="little").view("<u8")
    return np.ascontiguousarray(words).view(np.int64)
