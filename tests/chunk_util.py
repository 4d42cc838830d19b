"""Attention of new tokens over a paged INT4 cache in plain 64-bit arithmetic (test infrastructure: shares no code with the library)."""
import numpy as np

import paged_util as pu

E4M3 = pu.E4M3


def ranges(new, length, first=None, end=None, window=0):
    """[lo, hi) of each of a sequence's new rows, as include/fireq_chunk.h defines them."""
    out = []
    for i in range(new):
        pos = length - new + i
        lo = 0 if first is None else int(first[i])
        hi = pos + 1 if end is None else int(end[i])
        if window:
            lo = max(lo, pos - window + 1)
        out.append((max(lo, 0), min(hi, max(length, 0))))
    return out


def attention(q, q_scale, tokens, pos, lo, hi, out_scale, cap, slope):
    """(output [128], tolerance [128]) of one query row over tokens lo .. hi - 1.

    The tolerance is that of paged_util.attention, whose score error passes a tanh at most unchanged, with 2^-20 of the score for the tanh
    and its FP32 arguments, and 2^-20 of the bias (a distance counted from the row's nearest token, one product and one sum in FP32)."""
    K, V, kc, ks, vs = (x[lo:hi] for x in tokens)
    if hi <= lo:
        return np.zeros(128), np.zeros(128)
    qv = E4M3[q]
    f = float(q_scale) * out_scale
    s = K @ qv * f
    x = cap * np.tanh(s / cap) if cap else s
    d = np.abs(pos - np.arange(lo, hi))
    bias = slope * (d - d.min())
    z = x - bias
    p = np.exp(z - z.max())
    n = p.sum()
    o = p @ V / n
    worst = np.abs(qv[None, :] * (kc + 8)).max(1) * np.abs(ks[:, 0]) * f
    near = z > z.max() - 60                               # (further ones have no weight, whatever their bias's error)
    e = 2.0 ** -12 * worst + 2.0 ** -20 * (2 * np.abs(s) + np.abs(s).max() + bias * near + np.abs(z[near]).max() + 1)
    e = np.minimum(e, 1.0)
    vs = np.abs(vs[:, 0])
    tol = 2.0 ** -8 * np.abs(o) + ((p * (2.0 ** -11 + e)) @ np.abs(V) + (p * e).sum() * np.abs(o)) / n
    tol += 2.0 ** -25 * 2.0 ** -7 * 8 * (hi - lo) / n + 2.0 ** -19 * 16 * (p @ vs) / n
    return o, tol
