"""The KV cache held in 8 bits, restated on the CPU in 64 bits: what a write leaves in it, what a read gives, attention over it.

A cache is a list of sequences; a sequence's K (or V) is a dict with the integer codes or e4m3 values [capacity, Hkv, d], and
scales [blocks, Hkv], as float64 arrays."""
import math

import numpy as np
import torch

TINY = 2.0 ** -126


def scale_of(amax, code):
    """The fp32 number stored as the scale of a block with this largest magnitude, as a float64."""
    if not np.isfinite(amax):
        return math.nan
    if code == "int8":
        return max(float(np.float32(amax) / np.float32(127)), TINY)
    if amax == 0:
        return TINY
    k = math.frexp(amax / 448.0)[1]               # amax / 448 = m 2^k, 1/2 <= m < 1 (the division is exact where it matters:
    while amax <= 448.0 * 2.0 ** (k - 1):         # these two loops compare products of a power of two)
        k -= 1
    while amax > 448.0 * 2.0 ** k:
        k += 1
    return max(2.0 ** k, TINY)


def codes_of(x, scale, code):
    """Codes (as the numbers they are) of the float64 values x under one scale."""
    if math.isnan(scale):
        return np.zeros_like(x)
    y = x / scale                                  # (24 bits by 24 bits: a float64 quotient lies on the right side of every border)
    if code == "int8":
        return np.clip(np.rint(y), -127, 127)
    a = np.abs(y)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.sign(y) * np.rint(a / step) * step


class Side:
    """K or V of one sequence."""

    def __init__(self, capacity, Hkv, d, code, block):
        self.code, self.block = code, block
        self.codes = np.zeros((capacity, Hkv, d))
        self.scales = np.zeros((-(-capacity // block), Hkv))

    def write(self, x, start):
        """x: float64 [n, Hkv, d] (values of bf16 or fp32 numbers)."""
        n, blk = x.shape[0], self.block
        for j in range(start // blk, -(-(start + n) // blk) if n else 0):
            lo, hi = max(start, j * blk), min(start + n, (j + 1) * blk)
            for h in range(x.shape[1]):
                part = x[lo - start:hi - start, h]
                s = scale_of(np.abs(part).max() if np.isfinite(part).all() else math.inf, self.code)
                if lo > j * blk:
                    before = self.scales[j, h]
                    s = math.nan if math.isnan(s) or math.isnan(before) else max(before, s)
                    if s > before:
                        old = np.float32(self.codes[j * blk:lo, h]) * np.float32(before)      # what is read back, an fp32 number
                        self.codes[j * blk:lo, h] = codes_of(old.astype(np.float64), s, self.code)
                self.codes[lo:hi, h] = codes_of(part, s, self.code)
                self.scales[j, h] = s

    def read(self, start, n):
        """fp32 values."""
        at = np.arange(start, start + n)
        return np.float32(self.codes[at]) * np.float32(self.scales[at // self.block])[:, :, None]

    def values(self, n):
        """float64 values of tokens 0 .. n - 1."""
        return self.codes[:n] * self.scales[np.arange(n) // self.block][:, :, None]


def unpack(cache, name):
    """What the device holds, as Sides (codes exactly, whatever their strides)."""
    codes, scales = getattr(cache, name + "_codes"), getattr(cache, name + "_scales")
    code = {torch.int8: "int8", torch.float8_e4m3fn: "e4m3"}[codes.dtype]
    blk, out = cache.c.block_tokens, []
    host = codes.cpu().double().numpy()
    rows = scales.cpu().double().numpy()
    for b, n in enumerate(cache.lengths):
        t0 = int(cache.cu_host[b])
        s = Side(n, codes.shape[1], codes.shape[2], code, blk)
        s.codes = host[t0:t0 + n]
        s.scales = rows[t0 // blk + b:t0 // blk + b + s.scales.shape[0]]
        out.append(s)
    return out


def attention(q, K, V, keep, scale):
    """One query: q [d], K, V [n, d], keep bool [n]; float64.  Returns O [d], lse, and what bounds the kernel's error: the
    probability-weighted magnitude of V per dimension, the largest sum |q_i K_ji| * scale, the largest |V|, the keys."""
    d = q.shape[0]
    K, V = K[keep], V[keep]
    if K.shape[0] == 0:
        return np.zeros(d), -math.inf, np.zeros(d), 0.0, 0.0, 0
    x = scale * (K @ q)
    m = x.max()
    p = np.exp(x - m)
    l = p.sum()
    return p @ V / l, m + math.log(l), p @ np.abs(V) / l, float((np.abs(K) @ np.abs(q)).max() * scale), float(np.abs(V).max()), K.shape[0]


def tolerance(O, A, S, vmax, n, dtype):
    """How far O [d] may be off.  With A, S, vmax, n as above and u = 2^-24:
      logits     d products and sums in fp32 and three more roundings, a tensor-core sum rounded toward zero (2 u each): off by
                 (2 d + 8) u S + 2^-21 (exponential), twice that in O relative to A (numerator and denominator)
      weights    held as fp16 (2^-11 relative), or as the sum of two (2^-22); the step of fp16 below its normal range is 2^-24, and
                 neither one number nor the second of two is finer: off by 2^-25 of a unit that is at most vmax / 64 (the reference
                 keeps the largest weight of a scale above 64): n 2^-31 vmax
      sums       n / 16 tensor-core sums of 16 products, 2 u each, and the joining of warps and blocks, relative to A
      result     rounded once"""
    u, d = 2.0 ** -24, O.shape[0]
    bf16 = dtype == torch.bfloat16
    rel = 2 * ((2 * d + 8) * u * S + 2.0 ** -21) + (2.0 ** -11 if bf16 else 2.0 ** -22) + 2 * u * (n / 16 + 32)
    return rel * A + n * vmax * 2.0 ** -31 + np.abs(O) * (2.0 ** -8 if bf16 else u)


def lse_tolerance(lse, d, S, n):
    """(sums of the probabilities in fp32, lane by lane, then lanes, warps and blocks)"""
    u = 2.0 ** -24
    return (2 * d + 8) * u * S + 2.0 ** -21 + u * (n / 16 + 64) + 4 * u * abs(lse)


def weights(q, K, scales, keep, scale):
    """One query: the largest weight p_j * scales_j of its kept keys (p: probabilities; scales [n]: V's), and the sum of the
    weights; float64."""
    x = scale * (K[keep] @ q)
    p = np.exp(x - x.max())
    w = p / p.sum() * scales[keep]
    return float(w.max()), float(w.sum())


def tight_tolerance(O, A, S, wmax, code, n, dtype):
    """As `tolerance`, with what fp16's last step drops counted against the query's own weights: a weight is held in units in
    which the largest that its warp has seen for this query is 2^11 or more, off by 2^-25 of one, and takes a code of at most 127
    (int8) or 448 (e4m3); the second number of an fp32 weight is held 2^11 times larger.  wmax: the largest weight of all keys, n
    of them."""
    top = 127 if code == "int8" else 448
    return tolerance(O, A, S, 0.0, n, dtype) + n * top * wmax * 2.0 ** (-36 if dtype == torch.bfloat16 else -47)
