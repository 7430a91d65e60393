"""The rotation of queries and keys and the 4-bit cache by their definitions, in float64 (NumPy; test
infrastructure only).

4-bit form: e2m1 codes (1 sign, 2 exponent, 1 mantissa bit, bias 1), two a byte, the even channel in
the low half, and one scale byte e per 32 channels, value 2^(e - 127) (255: NaN)."""
import numpy as np

PAGE, BLOCK = 64, 32
POSITIVE = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([POSITIVE, -POSITIVE])


def encode(x):
    """Codes of float64 |x| <= 6: nearest, ties to the even code."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    hi = np.minimum(np.searchsorted(POSITIVE, a), 7)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - POSITIVE[lo], POSITIVE[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (c | np.where(np.signbit(x), 8, 0)).astype(np.uint8)


def scale_byte(amax):
    """The smallest e >= 1 with amax <= 6 * 2^(e - 127); 255 for what is not finite."""
    amax = np.asarray(amax, np.float64)
    ok = np.isfinite(amax)
    m, p = np.frexp(np.where(ok, amax, 1))  # amax = m 2^p, 0.5 <= m < 1; 6 = 0.75 * 2^3
    e = np.where(amax == 0, 1, p - 3 + np.where(m > 0.75, 1, 0) + 127)
    return np.where(ok, np.maximum(e, 1), 255).astype(np.uint8)


def scale_value(e):
    e = np.asarray(e)
    return np.where(e == 255, np.nan, np.exp2(e.astype(np.float64) - 127))


def quantise(x):
    """(bytes [..., dh / 2], scale bytes [..., ceil(dh / 32)]) of x [..., dh]."""
    x = np.asarray(x, np.float64)
    dh = x.shape[-1]
    b = np.zeros(x.shape[:-1] + (-(-dh // BLOCK) * BLOCK,))
    b[..., :dh] = x
    b = b.reshape(x.shape[:-1] + (-1, BLOCK))
    with np.errstate(invalid="ignore"):
        e = scale_byte(np.where(np.isnan(b), np.inf, np.abs(b)).max(-1))
    bad = (e == 255)[..., None]
    c = encode(np.where(bad, 0, b) / np.where(bad, 1, scale_value(e)[..., None]))
    c = np.where(bad, 0, c).astype(np.uint8).reshape(x.shape[:-1] + (-1,))[..., :dh]
    return c[..., ::2] | (c[..., 1::2] << 4), e


def values(codes, e):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    return VALUES[c] * np.repeat(scale_value(e), BLOCK, -1)[..., :c.shape[-1]]


def places(table, pos, count, T, n_pages):
    """(r, t, page, slot) of the tokens of a call that the cache has a place for."""
    for r in range(table.shape[0]):
        n = T if count is None else min(max(int(count[r]), 0), T)
        for t in range(n):
            at = int(pos[r]) + t
            if pos[r] >= 0 and at // PAGE < table.shape[1] and 0 <= table[r, at // PAGE] < n_pages:
                yield r, t, table[r, at // PAGE], at % PAGE


def append(x, codes, scales, table, pos, count=None):
    """x [R][T][H][dh] into copies of codes [P][H][64][dh / 2] and scales [P][H][64][blocks]."""
    codes, scales = codes.copy(), scales.copy()
    for r, t, page, slot in places(table, pos, count, x.shape[1], codes.shape[0]):
        codes[page, :, slot], scales[page, :, slot] = quantise(x[r, t])
    return codes, scales


def read(codes, scales, table, pos, T, count=None):
    """[R][T][H * dh]: zeros where nothing is held."""
    P, H, _, half = codes.shape
    out = np.zeros((table.shape[0], T, H, 2 * half))
    for r, t, page, slot in places(table, pos, count, T, P):
        out[r, t] = values(codes[page, :, slot], scales[page, :, slot])
    return out.reshape(table.shape[0], T, -1)


def row_of(codes, scales, table_row, n, head):
    """Values [n][dh] of a row's first n tokens of a head, and which of them are in a page."""
    out, there = np.zeros((n, 2 * codes.shape[3])), np.zeros(n, bool)
    for p in range(-(-n // PAGE)):
        page = table_row[p]
        if not 0 <= page < codes.shape[0]:
            continue
        m = min(PAGE, n - p * PAGE)
        out[p * PAGE:p * PAGE + m] = values(codes[page, head, :m], scales[page, head, :m])
        there[p * PAGE:p * PAGE + m] = True
    return out, there


def attention(q, kp, vp, ks, vs, table, lens, scale, kv_heads, qpos=None):
    """q [R][S][Hq][dh] -> (o, spread, size, most): o [R][S][Hq][dh]; spread = sum p |v| / sum p of
    each output, size = the largest sum |q k| |scale| of each query's scores, most = its largest
    |score| (for error bounds)."""
    R, S, Hq, dh = q.shape
    o, spread = np.zeros(q.shape), np.zeros(q.shape)
    size, most = np.zeros((R, S, Hq, 1)), np.zeros((R, S, Hq, 1))
    g = Hq // kv_heads
    for r in range(R):
        n = min(max(int(lens[r]), 0), table.shape[1] * PAGE)
        for h in range(kv_heads):
            k, there = row_of(kp, ks, table[r], n, h)
            v, _ = row_of(vp, vs, table[r], n, h)
            for i in range(S):
                lim = n if qpos is None else min(n, max(0, int(qpos[r]) + i + 1))
                see = there[:lim]
                if not see.any():
                    continue
                kk, vv = k[:lim][see], v[:lim][see]
                qq = np.asarray(q[r, i, h * g:(h + 1) * g], np.float64)
                a = qq @ kk.T * scale
                with np.errstate(invalid="ignore"):
                    p = np.exp(a - a.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o[r, i, h * g:(h + 1) * g] = p @ vv
                spread[r, i, h * g:(h + 1) * g] = p @ np.abs(vv)
                size[r, i, h * g:(h + 1) * g, 0] = (np.abs(qq) @ np.abs(kk).T).max(1) * abs(scale)
                most[r, i, h * g:(h + 1) * g, 0] = np.abs(a).max(1)
    return o, spread, size, most


def rope(x, pos, axes, freqs, w=None, eps=None, halves=False):
    """x [R][S][H][dh] -> (y, size): y normed and rotated; size[c] = |u| + |v| of the pair of c."""
    y = np.asarray(x, np.float64)
    if eps is not None:
        y = y / np.sqrt(np.mean(y * y, -1, keepdims=True) + eps) * (1 if w is None else w)
    out, size = y.copy(), np.abs(y)
    at = p = 0
    for a, n in enumerate(axes):
        h = n // 2
        angle = (pos[..., a:a + 1].astype(np.float64) * freqs[p:p + h])[:, :, None]
        u = slice(at, at + h) if halves else slice(at, at + n, 2)
        v = slice(at + h, at + n) if halves else slice(at + 1, at + n, 2)
        out[..., u] = y[..., u] * np.cos(angle) - y[..., v] * np.sin(angle)
        out[..., v] = y[..., v] * np.cos(angle) + y[..., u] * np.sin(angle)
        size[..., u] = size[..., v] = np.abs(y[..., u]) + np.abs(y[..., v])
        at, p = at + n, p + h
    return out, size
