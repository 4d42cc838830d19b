"""A paged INT4 key/value cache and its attention in plain 64-bit arithmetic on the CPU (test infrastructure: shares no code with
the library).  The cache's bytes are addressed one by one, as include/fireq_paged.h describes them."""
import functools

import numpy as np
import torch

TILE = 2080


def e4m3_values():
    """Value of each E4M3 code."""
    return torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()


E4M3 = e4m3_values()


def to_e4m3(x):
    """Codes of the nearest E4M3 numbers (ties to even) of float32 values; saturating, NaN to zero."""
    return torch.as_tensor(np.clip(np.asarray(x, np.float32), -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def key_place(t, d):
    """(byte in the head's page, high nibble?) of dimension d of token t's key."""
    return t // 16 * TILE + 256 * (d // 32) + 16 * (t % 16) + d % 16, d // 16 % 2


def value_place(t, c):
    return t // 16 * TILE + 1024 + 256 * (t % 16 // 4) + 16 * (c % 16) + 4 * (c // 32) + (0, 2, 1, 3)[t % 4], c // 16 % 2


def scale_place(t, value):
    return t // 16 * TILE + 2048 + 8 * (t % 16 // 4) + t % 4 + (4 if value else 0)


@functools.lru_cache(maxsize=None)
def places(t, value):
    """Bytes and shifts of the 128 codes of token t."""
    at = [(value_place if value else key_place)(t, d) for d in range(128)]
    return np.array([p for p, _ in at]), 4 * np.array([h for _, h in at])


class Cache:
    """numpy uint8 [pages, heads, page / 16, 2080] with token access."""

    def __init__(self, pages, heads, page, rng, stale_nan=True):
        self.b = rng.integers(0, 256, (pages, heads, page // 16, TILE), dtype=np.uint8)
        if stale_nan:                                     # what was never appended must not count: NaN scales
            self.b[..., 2048:] = 0x7F
        self.page = page

    def flat(self, p, h):
        return self.b[p, h].reshape(-1)

    def put(self, slot, h, value, codes, scale):
        row, t = self.flat(slot // self.page, h), slot % self.page
        at, sh = places(t, value)
        n = (np.asarray(codes) + 8).astype(np.uint8)
        for half in (0, 4):                               # (a byte holds two dimensions)
            on = sh == half
            row[at[on]] = (row[at[on]] & (0xF0 >> half)) | (n[on] << half)
        row[scale_place(t, value)] = scale

    def get(self, slot, h, value):
        """(codes int [128], E4M3 scale code)"""
        row, t = self.flat(slot // self.page, h), slot % self.page
        at, sh = places(t, value)
        return (row[at] >> sh & 15).astype(int) - 8, int(row[scale_place(t, value)])

    def tokens(self, slots, h):
        """64-bit (keys, values) [n, 128] and the key codes and scales they come from."""
        K, V, kc, ks, vs = [], [], [], [], []
        for s in slots:
            c, sc = self.get(int(s), h, False)
            K.append(c * E4M3[sc])
            kc.append(c)
            ks.append(E4M3[sc])
            c, sc = self.get(int(s), h, True)
            V.append(c * E4M3[sc])
            vs.append(E4M3[sc])
        return (np.array(x, np.float64).reshape(len(slots), n) for x, n in ((K, 128), (V, 128), (kc, 128), (ks, 1), (vs, 1)))


def int4(x):
    """(codes, E4M3 scale code) of one float32 head."""
    x = np.asarray(x, np.float32)
    sc = int(to_e4m3(min(np.float32(np.abs(x).max()) / np.float32(7), np.float32(448))))
    s = np.float32(E4M3[sc])
    if s == 0:
        return np.zeros(128, int), sc
    return np.clip(np.rint(x / s), -8, 7).astype(int), sc


def rotate(x, cs, interleaved):
    """float32 [128] -> rotated, products and sums in 64 bits, rounded once."""
    x = np.asarray(x, np.float64)
    c, s = np.asarray(cs, np.float64).T
    o = np.empty(128)
    a, b = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, 64), slice(64, 128))
    o[a] = x[a] * c - x[b] * s
    o[b] = x[b] * c + x[a] * s
    return o.astype(np.float32)


def attention(q, q_scale, K, V, kc, ks, vs, out_scale):
    """(output [128], tolerance [128]) of one query over tokens, in 64 bits.

    The tolerance counts, per element: half a bf16 step (2^-8); the probabilities' rounding to fp16 (2^-11 each, or half a fp16
    subnormal step, 2^-25, relative to 2^7 times the largest, times sigma); the scores' error, of an FP8 product that adds with 2^-13 relative to the
    largest term of the zero-point form, plus 2^-20 of the score for its FP32 factors, which moves a probability by as
    much; and FP32 sums of the value codes with their zero point, 2^-19 of sum p sigma 16."""
    qv = E4M3[q]
    if len(K) == 0:
        return np.zeros(128), np.zeros(128)
    f = float(q_scale) * out_scale
    s = K @ qv * f
    p = np.exp(s - s.max())
    n = p.sum()
    o = p @ V / n
    worst = np.abs(qv[None, :] * (kc + 8)).max(1) * np.abs(ks[:, 0]) * f
    e = 2.0 ** -12 * worst + 2.0 ** -20 * (np.abs(s) + np.abs(s.max()) + 1)
    vs = np.abs(vs[:, 0])
    tol = 2.0 ** -8 * np.abs(o) + ((p * (2.0 ** -11 + e)) @ np.abs(V) + (p * e).sum() * np.abs(o)) / n
    tol += 2.0 ** -25 * 2.0 ** -7 * 8 * len(K) / n + 2.0 ** -19 * 16 * (p @ vs) / n
    return o, tol
