"""The 8-bit operators by their definitions, in float64 (NumPy; test infrastructure only).

8-bit form: e4m3 codes (1 sign, 4 exponent, 3 mantissa bits, bias 7, largest 448, 0x7F NaN) and
one scale byte e per block, value 2^(e - 127) (255: NaN)."""
import numpy as np

PAGE = 64


def _table():
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(c & 127) == 127] = np.nan
    return np.where(c >= 128, -v, v)


VALUES = _table()


def encode(x):
    """Codes of float64 x, |x| <= 448 or NaN: nearest, ties to the even mantissa."""
    x = np.asarray(x, np.float64)
    a = np.abs(np.where(np.isnan(x), 0, x))
    pos = VALUES[:127]
    hi = np.minimum(np.searchsorted(pos, a), 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = np.where(np.isnan(x), 127, c)
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_byte(amax):
    """The smallest e >= 1 with amax <= 448 * 2^(e - 127)."""
    amax = np.asarray(amax, np.float64)
    m, p = np.frexp(amax)  # amax = m 2^p, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = np.where(amax == 0, 1, p - 9 + np.where(m > 0.875, 1, 0) + 127)
    return np.maximum(e, 1).astype(np.uint8)


def scale_value(e):
    e = np.asarray(e)
    return np.where(e == 255, np.nan, np.exp2(e.astype(np.float64) - 127))


def _finite(x):
    return np.where(np.isfinite(x), x, 0)


def quantise(x, rows=1):
    """(codes [M][K], scale bytes [ceil(M / rows)][ceil(K / 128)]) of x [M][K]."""
    x = np.asarray(x, np.float64)
    M, K = x.shape
    b = np.zeros((-(-M // rows) * rows, -(-K // 128) * 128))
    b[:M, :K] = x
    b = b.reshape(-1, rows, b.shape[1] // 128, 128)
    s = scale_byte(np.abs(_finite(b)).max((1, 3)))
    q = encode(np.where(np.isfinite(b), b, np.nan) / scale_value(s)[:, None, :, None])
    return q.reshape(-1, b.shape[2] * 128)[:M, :K].copy(), s


def values(q, s, rows=1):
    M, K = q.shape
    f = np.repeat(np.repeat(scale_value(s), rows, 0)[:M], 128, 1)[:, :K]
    return VALUES[q] * f


def rmsnorm(x, w, r=None, eps=1e-6):
    s = np.asarray(x, np.float64) + (0 if r is None else np.asarray(r, np.float64))
    return s / np.sqrt(np.mean(s * s, 1, keepdims=True) + eps) * np.asarray(w, np.float64)


def append(x, codes, scales, table, pos, count, transposed):
    """x [R][T][H][dh] into copies of codes ([P][H][64][dh], or [P][H][dh][64] if transposed) and
    scales [P][H]: (codes, scales)."""
    codes, scales = codes.copy(), scales.copy()
    R, T, H, _ = x.shape
    for r in range(R):
        n = min(max(int(count[r]), 0), T)
        first = int(pos[r])
        if first < 0 or n == 0:
            continue
        for p in range(first // PAGE, (first + n - 1) // PAGE + 1):
            if p >= table.shape[1] or not 0 <= table[r, p] < codes.shape[0]:
                continue
            page = table[r, p]
            lo, hi = max(first, p * PAGE), min(first + n, (p + 1) * PAGE)
            a, b = lo - p * PAGE, hi - p * PAGE
            for h in range(H):
                new = np.asarray(x[r, lo - first:hi - first, h], np.float64)
                e = int(scale_byte(np.abs(_finite(new)).max()))
                c = codes[page, h].T if transposed else codes[page, h]  # a view [64][dh]
                if a > 0:
                    old = int(scales[page, h])
                    if e > old:
                        c[:a] = encode(VALUES[c[:a]] * 2.0 ** (old - e))
                    e = max(e, old)
                scales[page, h] = e
                c[a:b] = encode(np.where(np.isfinite(new), new, np.nan) * 2.0 ** (127 - e))
    return codes, scales


def read_cache(codes, scales, table_row, n, head, transposed):
    """Values [n][dh] of a row's first n tokens of a head, and which of them are in a page."""
    dh = codes.shape[2] if transposed else codes.shape[3]
    out, there = np.zeros((n, dh)), np.zeros(n, bool)
    for p in range(-(-n // PAGE)):
        page = table_row[p]
        if not 0 <= page < codes.shape[0]:
            continue
        c = codes[page, head].T if transposed else codes[page, head]
        m = min(PAGE, n - p * PAGE)
        out[p * PAGE:p * PAGE + m] = VALUES[c[:m]] * scale_value(scales[page, head])
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
            k, there = read_cache(kp, ks, table[r], n, h, False)
            v, _ = read_cache(vp, vs, table[r], n, h, True)
            for i in range(S):
                lim = n if qpos is None else min(n, max(0, int(qpos[r]) + i + 1))
                see = there[:lim]
                if not see.any():
                    continue
                kk, vv = k[:lim][see], v[:lim][see]
                qq = np.asarray(q[r, i, h * g:(h + 1) * g], np.float64)
                a = qq @ kk.T * scale
                p = np.exp(a - a.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o[r, i, h * g:(h + 1) * g] = p @ vv
                spread[r, i, h * g:(h + 1) * g] = p @ np.abs(vv)
                size[r, i, h * g:(h + 1) * g, 0] = (np.abs(qq) @ np.abs(kk).T).max(1) * abs(scale)
                most[r, i, h * g:(h + 1) * g, 0] = np.abs(a).max(1)
    return o, spread, size, most
