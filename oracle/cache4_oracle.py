"""fp64 CPU oracle for the KV cache in 4 bits and the attention over it.

TEST INFRASTRUCTURE ONLY, like the rest of ``oracle/``: it shares no code with
the HIP path.

* ``quantise4_ref`` -- codes and scale bytes of bf16 rows: groups of 32 along
  the last axis share 2^(b - 127); a group with largest magnitude a takes the
  smallest e in -120 .. 125 with a <= 7 * 2^e (e = 125 where none has it),
  b = e + 127; elements x / 2^e go to the nearest of the eight magnitudes, ties
  to the even code, past 6 to 6, the sign kept; a group with an infinity or a NaN
  gets b = 255 and codes of zero.
* ``values4_ref`` -- what codes and scale bytes stand for.
* ``decode4_ref`` -- attention of the new tokens over the first ``cache_len``
  rows; causal: the last n_new of them are the new tokens' own.

Every function is pinned by ``tests/test_cache4_pins.py``.
"""
from __future__ import annotations

import math

import numpy as np

from .apb_oracle import bf16_to_f64

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def quantise4_ref(bits):
    """bf16 bits [.., d] -> codes uint8 [.., d / 2], scale bytes uint8 [.., d / 32]."""
    bits = np.asarray(bits, dtype=np.uint16)
    x = bf16_to_f64(bits).reshape(bits.shape[:-1] + (-1, 32))
    negative = (bits >> 15).reshape(x.shape)
    bad = ~np.isfinite(x).all(-1)
    a = np.abs(np.where(bad[..., None], 0.0, x))
    top = a.max(-1)
    e = np.full(top.shape, 125)
    for cand in range(124, -121, -1):
        e = np.where(top <= 7.0 * 2.0 ** cand, cand, e)
    y = a / np.exp2(e.astype(np.float64))[..., None]
    # distance to every magnitude; the even codes are asked first, so that they
    # keep a tie
    order = [0, 2, 4, 6, 1, 3, 5, 7]
    far = np.stack([np.abs(y - MAGNITUDES[c]) for c in order])
    code = np.array(order, dtype=np.uint8)[far.argmin(0)]
    code = code | (negative << 3).astype(np.uint8)
    code = np.where(bad[..., None], 0, code).astype(np.uint8).reshape(bits.shape)
    scale = np.where(bad, 255, e + 127).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def values4_ref(codes, scales):
    """fp64 values [.., d] of codes [.., d / 2] and scale bytes [.., d / 32]."""
    codes = np.asarray(codes, dtype=np.uint8)
    code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    level = np.array(MAGNITUDES + tuple(-m for m in MAGNITUDES))[code]
    by = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (level.reshape(scales.shape + (32,)) * by[..., None]).reshape(code.shape)


def decode4_ref(q, k, v, *, causal, scale=None, bound=False):
    """fp64 attention of q [n_q, n_new, d] (bf16 bits) over the rows k, v [n_kv,
    cache_len, d] (fp64 values).  Returns (o, lse); rows that see no key get 0 and
    -inf, and keys that a row does not see have no part in it.  With ``bound`` also
    sum p |v| [n_q, n_new, d] and the largest scale * sum |q_i k_i| over a row's
    visible keys [n_q, n_new], which error bounds are made of."""
    n_q, n_new, d = q.shape
    n_kv, keys, _ = k.shape
    g = n_q // n_kv
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    qf = bf16_to_f64(q)
    o, lse = np.zeros((n_q, n_new, d)), np.full((n_q, n_new), -np.inf)
    pv, qk = np.zeros((n_q, n_new, d)), np.zeros((n_q, n_new))
    for h in range(n_q):
        for j in range(n_new):
            end = keys - n_new + j + 1 if causal else keys
            if end < 1:
                continue
            kh, vh = k[h // g, :end], v[h // g, :end]
            s = kh @ qf[h, j] * scale
            m = s.max()
            p = np.exp(s - m)
            total = p.sum()
            o[h, j] = p @ vh / total
            lse[h, j] = m + np.log(total)
            if bound:
                pv[h, j] = p @ np.abs(vh) / total
                qk[h, j] = (np.abs(kh) @ np.abs(qf[h, j])).max() * scale
    return (o, lse, pv, qk) if bound else (o, lse)
