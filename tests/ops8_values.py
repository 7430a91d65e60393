"""Caches whose values or scores lie far apart, and how far attention over them may be off.

Bound of an output o = sum p v / sum p (p relative to the row's largest probability, so sum p >= 1;
E = 2^-23 a float32 operation, u(t) one rounding to t):
  scores         dh float32 additions and three products, the shift by the reference, the exponential:
                 dh E sum |q k| + 8 E |score| + 4 E of p, in numerator and denominator: twice of sum p |v|
  probabilities  rounded to float16, the same rounded ones above and below: u(float16) p each, twice, or
                 where p is subnormal there 2^-25 of a reference that is 2^9 below the largest p or less:
                 2^-34, of sum |v| above and of n |o| below
  sums           n terms in float32: n E of sum p |v|; sums that are kept in the unit of the largest
                 value scale that the query sees: 2^-149 of that scale for each of n terms
  result         u(t) |o|, and 2^-25 where a float16 result is subnormal (2^-134: bfloat16)
"""
import numpy as np

from oracle import ops8 as O

E = 2.0 ** -23
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def seen_values(pages, table, lens, S, Hq, qpos=None):
    """Of each query: sum |v| of the tokens it sees [R][S][Hq][dh], and its largest value scale."""
    kp, vp, ks, vs = pages
    R, H, dh = table.shape[0], kp.shape[1], kp.shape[3]
    reach, top = np.zeros((R, S, Hq, dh)), np.zeros((R, S, Hq, 1))
    for r in range(R):
        n = min(max(int(lens[r]), 0), table.shape[1] * 64)
        for h in range(H):
            v, there = O.read_cache(vp, vs, table[r], n, h, True)
            scale = np.where(there, np.repeat([O.scale_value(vs[p, h]) if 0 <= p < len(vs) else 0
                                               for p in table[r]], 64)[:n], 0)
            total = np.vstack([np.zeros(dh), np.cumsum(np.abs(v) * there[:, None], 0)])
            most = np.concatenate([[0.0], np.maximum.accumulate(scale)]) if n else np.zeros(1)
            for i in range(S):
                lim = n if qpos is None else min(n, max(0, int(qpos[r]) + i + 1))
                g = slice(h * Hq // H, (h + 1) * Hq // H)
                reach[r, i, g], top[r, i, g] = total[lim], most[lim]
    return reach, top


def attention(q, pages, table, lens, scale, qpos=None, dtype="bf16"):
    """(o, bound) of q [R][S][Hq][dh] (float64)."""
    R, S, Hq, dh = q.shape
    o, spread, size, most = O.attention(q, *pages, table, lens, scale, pages[0].shape[1], qpos)
    reach, top = seen_values(pages, table, lens, S, Hq, qpos)
    n = table.shape[1] * 64
    rel = 2 * (dh * E * size + 8 * E * most + 4 * E) + 2 * U["f16"] + n * E
    tol = rel * spread + 2.0 ** -34 * (reach + n * np.abs(o)) + n * 2.0 ** -149 * top
    tol = tol * (1 + U[dtype]) + U[dtype] * np.abs(o) + (2.0 ** -25 if dtype == "f16" else 2.0 ** -134)
    return o, tol


def codes(rng, shape, lo, hi):
    """Codes of either sign and of magnitudes from code lo to code hi - 1."""
    return (rng.integers(lo, hi, shape) | (rng.integers(0, 2, shape) << 7)).astype(np.uint8)


# Scale bytes of a row's value pages.  The largest comes first, last and between the others, which are
# `d` below it: within what a float16 operand holds beside it, past that, and as far as float32 sums
# reach.  (Four waves may take a row's pages in turn: the far ones are four apart.)
DISTANCES = (5, 6, 7, 8, 9, 20, 40, 64, 65, 79, 80, 81, 100, 113, 114, 120)
ORDERS = {"first": (0, 1, 1, 1, 1), "last": (1, 1, 1, 1, 0), "middle": (1, 1, 1, 1, 0, 1, 1, 1, 1)}


def far_cache(d, order, dh=64, top=200, seed=0):
    """One row and one head: pages with 1 in ORDERS[order] have value scales d below the one with 0, whose
    codes are zero in half of the channels: the others decide those outputs."""
    rng = np.random.default_rng(seed + d)
    W = len(ORDERS[order])
    table = rng.permutation(W + 2)[:W].reshape(1, W).astype(np.int32)
    P = W + 2
    kp, vp = codes(rng, (P, 1, 64, dh), 0x20, 0x40), codes(rng, (P, 1, dh, 64), 0x28, 0x38)
    ks, vs = np.full((P, 1), 125, np.uint8), np.full((P, 1), 255, np.uint8)
    for j, below in enumerate(ORDERS[order]):
        vs[table[0, j]] = top - d * below
        if not below:
            vp[table[0, j], :, :dh // 2] = 0
    return [kp, vp, ks, vs], table


def queries(S, heads, dh, seed=1):
    return np.random.default_rng(seed).integers(-16, 17, (1, S, heads, dh)) / 16.0


# One key 2^bits above all others in the sum, its value zero; scores of the others up to `spread` powers
# of two apart.
TAILS = [(20.0, 0.0), (25.1, 0.0), (24.5, 0.5), (24.5, 1.0), (28.0, 0.0)]


def tail_cache(S, at, bits, spread, W=160, dh=64):
    """(q, pages, table, tokens, scale) of one row and head with the large key at token `at`."""
    rng = np.random.default_rng(3)
    table = rng.permutation(W).reshape(1, W).astype(np.int32)
    kp = np.zeros((W, 1, 64, dh), np.uint8)
    q = np.zeros((1, S, 1, dh))
    q[..., 0] = 1
    if spread:
        kp[:, 0, :, 1:] = codes(rng, (W, 64, dh - 1), 0x10, 0x20)
        q[..., 1:] = rng.integers(-8, 9, (1, S, 1, dh - 1)) * (spread / 8)
    vp = rng.integers(0x38, 0x48, (W, 1, dh, 64)).astype(np.uint8)     # 1 .. 4
    kp[table[0, at // 64], 0, at % 64, 0] = 0x7E                       # 448
    vp[table[0, at // 64], 0, :, at % 64] = 0
    pages = [kp, vp, np.full((W, 1), 127, np.uint8), np.full((W, 1), 131, np.uint8)]
    return q, pages, table, W * 64 - 5, bits * np.log(2) / 448
