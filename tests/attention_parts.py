"""Rows of attention over 8-bit codes whose roundings line up, with a bound for each element (numpy; test infrastructure).

What the kernel computes of a row of n cells, with u = 2^-24 (2 u where a matrix core may cut off), |x| magnitudes and
a_j = |scale| sum_d |q_d k_jd|:
  - score j: fp32 sums of dh exact products, twice as many where q goes through two bf16 parts, and four roundings
    around them: a_j (dh or 2 dh, + 4) 2 u.  Two parts leave 2^-17 of what they stand for (the first is off by at most half its
    unit, 2^-8 of the number's power of two; the rest is below that, and half a unit of its own eight bits is 2^-9 of a
    power of two at most 2^-8 there): a_j 2^-17 more.
  - weight j, w_j = e^(z_j - max): the exponential 2^-23; of its argument's roundings 16 u max a; for each of T steps of 256 cells
    and the joins behind them (4) another exponential and product, 2^-22.
  - p_j times its block's scale (exact) in two bf16 parts: 2^-17.
  - sums: 128 T additions of a wave's steps, 300 for the waves' and ranges' joins, 2 u each; the weights' own sum likewise.
So element d of the output o = sum w v / sum w is off by
  sum_j w_j |v_jd| (e_j + 2^-17) / L + |o_d| sum_j w_j e_j / L,   e_j the sum of all but the parts of p,
and by its own rounding: 2^-8 |o_d| in bf16, u |o_d| in fp32."""
import math

import numpy as np

U = 2.0 ** -24


def to_bf16(x):
    """x (fp32) to the nearest bf16, ties to even, as fp32."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def cut_bf16(x):
    """x (fp32) cut off to bf16, as fp32."""
    return (np.asarray(x, np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32)


def row(q, K, V, scale, io_bf16):
    """Output of one query over the cells K, V [n][dh] in 64 bits, and what each element may be off by."""
    q, K, V = (np.asarray(x, np.float64) for x in (q, K, V))
    n, dh = K.shape
    z, a = (K * q).sum(1) * scale, np.abs(K * q).sum(1) * abs(scale)
    w = np.exp(z - z.max())
    L = w.sum()
    o = (w[:, None] * V).sum(0) / L
    T = -(-n // 256)
    e = a * ((dh if io_bf16 else 2 * dh) + 4) * 2 * U + (0.0 if io_bf16 else a * 2.0 ** -17)
    e = e + 2.0 ** -23 + (T + 4) * 2.0 ** -22 + 16 * U * a.max() + (128 * T + 300) * 2 * U
    off = (w[:, None] * np.abs(V) * (e + 2.0 ** -17)[:, None]).sum(0) / L + np.abs(o) * (w * e).sum() / L
    return o, 1.01 * off + np.abs(o) * (2.0 ** -8 if io_bf16 else U) + 1e-30


def emulate(q, K, V, scale, io_bf16, plant=None):
    """The same with the kernel's roundings: operands in bf16 parts, fp32 between.  plant: a mistake, "q in one part",
    "p in one part" or "p cut off"."""
    q, K, V = (np.asarray(x, np.float32) for x in (q, K, V))
    qh = to_bf16(q)
    ql = np.zeros_like(q) if io_bf16 or plant == "q in one part" else to_bf16(q - qh)
    d = (K.astype(np.float64) @ qh + K.astype(np.float64) @ ql).astype(np.float32)
    s = d * np.float32(scale * math.log2(math.e))
    p = np.exp2(s - s.max()).astype(np.float32)
    ph, pl = (cut_bf16(p), None) if plant == "p cut off" else (to_bf16(p), None)
    pl = np.zeros_like(p) if plant in ("p in one part", "p cut off") else to_bf16(p - ph)
    o = ((ph.astype(np.float64) + pl) @ V.astype(np.float64)).astype(np.float32) / p.astype(np.float64).sum()
    return (to_bf16(o) if io_bf16 else o.astype(np.float32)).astype(np.float64)


MISTAKES = {True: ("p in one part", "p cut off"), False: ("p in one part", "p cut off", "q in one part")}

# magnitudes of codes that both formats hold
_MAGS = {"i8": np.arange(1, 128), "e4m3": np.unique(np.concatenate([np.arange(8, 16) * 2.0 ** e for e in range(-3, 4)]))}


def _balance(w, sign, code, r):
    """Codes with these signs whose sum with weights w is as near to zero as single steps bring it."""
    mags = _MAGS[code]
    at = r.randint(np.searchsorted(mags, 60), len(mags), len(w))
    total = lambda: float((w * sign * mags[at]).sum())  # noqa: E731
    for _ in range(4000):
        t = total()
        # all steps of one code, up or down: the one that leaves the least
        best = None
        for step in (-1, 1):
            to = np.clip(at + step, 0, len(mags) - 1)
            left = np.abs(t + w * sign * (mags[to] - mags[at]))
            j = int(left.argmin())
            if best is None or left[j] < best[0]:
                best = (left[j], j, to[j])
        if best[0] >= abs(t):
            break
        at[best[1]] = best[2]
    return sign * mags[at]


def aligned_case(code, dh, io_bf16, n, seed):
    """One query [dh] (fp32; of bf16 values if io_bf16) and codes of n <= 64 cells, K and V [n][dh], with a scale for all
    of each: sums that nearly vanish, but whose roundings do not if one of MISTAKES is made.
      V dims by quarters: the sign of what one bf16 part leaves of p; of what cutting p off leaves, about its median;
      all positive; the sign of what q's first part leaves of the score (cells in two halves)."""
    r = np.random.RandomState(seed)
    q = (r.randn(dh) * 1.5).astype(np.float32)
    if io_bf16:
        q = to_bf16(q)
    rest = np.sign((q - to_bf16(q)).astype(np.float64))
    if io_bf16:
        rest = np.where(r.rand(dh) < 0.5, 1.0, -1.0)
    half = np.where(np.arange(n) % 2 == 0, 1.0, -1.0)
    K = np.where(rest == 0, 1.0, rest)[None, :] * half[:, None] * np.where(r.rand(n, dh) < 0.15, -1.0, 1.0) * 64
    ks, vs, scale = 2.0 ** -7, 2.0 ** -3, 1 / math.sqrt(dh)
    z = (K * ks * q.astype(np.float64)).sum(1) * scale
    p = np.exp(z - z.max())
    p32 = p.astype(np.float32)
    kept = p - to_bf16(p32)
    cut = (p - cut_bf16(p32)) / p
    V = np.empty((n, dh))
    for d in range(dh):
        sign = [np.where(kept >= 0, 1.0, -1.0), np.where(cut >= np.median(cut), 1.0, -1.0), np.ones(n), half][4 * d // dh]
        if 4 * d // dh == 2:
            V[:, d] = _MAGS[code][r.randint(0, len(_MAGS[code]), n)]
        else:
            V[:, d] = _balance(p, sign, code, r)
    return q, K, ks, V, vs, scale
