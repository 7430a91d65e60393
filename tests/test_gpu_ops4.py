"""The rotation of queries and keys and the 4-bit cache against their float64 oracle.

Bounds.  u(t) = torch.finfo(t).eps / 2 is one rounding to t, E = 2^-23 one float32 operation (a
whole step: the matrix unit's own rounding of its sums is not specified to be to nearest).
  codes       scaling by a power of two is exact, so codes, scales and values read are the oracle's
              to the bit
  rope        the mean of squares takes 8 additions in a lane and at most 5 between lanes, a product
              and the division: 15 E, halved by the root, and root, division and two products:
              12 E of y.  An angle in turns is a float64 number of at most 2^31 radians (three
              roundings of 2^-53 of it: 2^-20.4 radians there, 10 E; nothing at the positions of the other
              tests), then a float32 one below 1 (2^-24 turns: 4 E in radians); its cosine and sine
              2 E; two products and a sum 2 E: 8 E + 10 E of |u| + |v|; one rounding u(t), and half
              the least subnormal of float16
  attention   a score is dh float32 additions and three products: (dh E sum |q k| + 4 E |score|)
              absolute, the shift by the reference and the exponential 4 E |score| + 4 E; twice that
              (numerator and sum) is a probability's relative error; its rounding to float16 is
              2^-11 relative, in numerator and sum, or 2^-34 of the query's largest where it is
              subnormal; sums of n terms in float32: n E; all of sum p |v|, and one rounding
              u(t) of the result
"""
import numpy as np
import pytest
import torch

from oracle import ops4 as O
from ops4_sizes import PLAN_SIZES

pytestmark = pytest.mark.gpu

E = 2.0 ** -23
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def u(t):
    return torch.finfo(t).eps / 2


def np64(t):
    return t.double().cpu().numpy()


def bits(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def rand(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype))).cuda()


def i32(a):
    return dev(a, np.int32)


def nv():
    import paper_2312_04429_amd as P
    return P


# -------------------------------------------------------------------------------------- rope

def check_rope(q, k, dh, pos, axes, qw=None, kw=None, eps=1e-6, halves=False, freqs=None, **kws):
    """q, k device [R][S][heads * dh]; pos NumPy [R][S][axes]."""
    if freqs is None:
        freqs = nv().nv_rope_freqs(axes)
    pd = i32(pos)
    got = nv().nv_op_qk_rope(q, k, dh, pd, axes, freqs, q_weight=qw, k_weight=kw, eps=eps, halves=halves,
                             **kws)
    for x, w, y in ((q, qw, got[0]), (k, kw, got[1])):
        if x is None:
            assert y is None
            continue
        R, S, C = x.shape
        with np.errstate(invalid="ignore", over="ignore"):
            want, size = O.rope(np64(x).reshape(R, S, C // dh, dh), np.asarray(pos), axes, np64(freqs),
                                None if w is None else np64(w), eps, halves)
        g = np64(y).reshape(want.shape)
        tol = 30 * E * size + u(x.dtype) * np.abs(want) + (2.0 ** -25 if x.dtype == F16 else 0)
        assert np.array_equal(np.isnan(g), np.isnan(want))
        with np.errstate(invalid="ignore"):
            bad = np.abs(g - want) > tol
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(),
                               float(np.nanmax(np.abs(g - want) / tol)))
    return got


AXES = {8: [(8,), (2, 2, 4)], 16: [(16,), (4, 6, 6)], 24: [(24,), (10, 14)], 32: [(32,), (0, 16, 16)],
        40: [(40,), (12, 14, 14)], 64: [(32,), (16, 24, 24)], 80: [(80,), (26, 26, 28)],
        128: [(128,), (44, 42, 42), (2, 30, 32, 64)], 136: [(136,), (40, 48, 48)],
        160: [(80,), (52, 54, 54)], 256: [(256,), (64, 96, 96)]}


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dh", sorted(AXES))
def test_rope(dh, halves, dtype):
    rng = np.random.default_rng(dh)
    for axes in AXES[dh]:
        for R, S, Hq, H in ((1, 1, 1, 1), (3, 5, 4, 2), (2, 67, 3, 3), (40, 1, 8, 1)):
            print("rope", dh, halves, dtype, axes, R, S, Hq, H, flush=True)
            q, k = rand(S, R, S, Hq * dh, dtype=dtype, scale=3.0), rand(S + 1, R, S, H * dh, dtype=dtype)
            pos = rng.integers(-1000, 200_000, (R, S, len(axes)))
            qw, kw = 1 + 0.2 * rand(1, dh), 1 + 0.2 * rand(2, dh)
            check_rope(q, k, dh, pos, axes, qw, kw, halves=halves)
            check_rope(q, k, dh, pos, axes, eps=None, halves=halves)
            check_rope(q, None, dh, pos, axes, None, None, halves=halves)
            check_rope(q, k, dh, pos, axes, None, kw, eps=0.5, halves=halves)


@pytest.mark.parametrize("halves", [False, True])
def test_rope_without_axes_is_the_norm(halves):
    q, k = rand(1, 2, 9, 4 * 64, dtype=F16), rand(2, 2, 9, 64, dtype=F16)
    check_rope(q, k, 64, np.zeros((2, 9, 0)), (), 1 + 0.2 * rand(1, 64), None, halves=halves)
    check_rope(q, k, 64, np.ones((2, 9, 2)), (0, 0), halves=halves)
    y = nv().nv_op_qk_rope(q, k, 64, i32(np.zeros((2, 9, 1))), (64,), nv().nv_rope_freqs((64,)),
                           eps=None, halves=halves)
    assert torch.equal(y[0], q) and torch.equal(y[1], k)  # position 0


@pytest.mark.parametrize("halves", [False, True])
def test_rope_views_of_one_product_and_in_place(halves):
    """Strided, unaligned and broadcast inputs, positions shared by rows; outputs that are inputs."""
    R, S, dh, axes = 3, 11, 64, (16, 48)
    pos = np.random.default_rng(1).integers(0, 99, (1, S, 2)).repeat(R, 0)
    for dtype, at, extra in ((F16, 0, 0), (BF16, 3, 7), (F16, 64, 8)):
        qkv = rand(5, R, S, 8 * dh + extra, dtype=dtype)
        q, k = qkv[:, :, at:at + 4 * dh], qkv[:, :, at + 4 * dh:at + 6 * dh]
        want = check_rope(q, k, dh, pos, axes, halves=halves)
        shared = i32(pos[:1]).expand(R, S, 2)
        freqs = nv().nv_rope_freqs(axes)
        got = nv().nv_op_qk_rope(q, k, dh, shared, axes, freqs, halves=halves)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        every = qkv.clone()
        other = every.clone()
        qq, kk = every[:, :, at:at + 4 * dh], every[:, :, at + 4 * dh:at + 6 * dh]
        back = nv().nv_op_qk_rope(qq, kk, dh, shared, axes, freqs, halves=halves, out=(qq, kk))
        assert back[0] is qq and torch.equal(qq, want[0]) and torch.equal(kk, want[1])
        every[:, :, at:at + 6 * dh] = other[:, :, at:at + 6 * dh]
        assert torch.equal(every, other)  # nothing beside the heads
        one = q[:1].expand(R, S, 4 * dh)
        check_rope(one, None, dh, pos, axes, halves=halves)


def test_rope_far_positions_and_any_frequencies():
    pos = np.array([2 ** 31 - 1, -2 ** 31, 12345678, 0, 1, 199_999])[None, :, None]
    for dtype in (F16, BF16):
        q = rand(3, 1, 6, 2 * 128, dtype=dtype)
        check_rope(q, None, 128, pos, (128,), eps=None)
        check_rope(q, q, 128, pos, (128,), halves=True)
    f = dev(np.random.default_rng(0).uniform(0, 1, 32), np.float64)
    check_rope(rand(4, 1, 6, 64, dtype=F16), None, 64, pos, (64,), freqs=f, eps=None)


def test_rope_values_that_are_not_ordinary():
    """Zero heads, heads of one large value, the types' smallest; what is not finite stays in its head."""
    for dtype in (F16, BF16):
        q = rand(6, 2, 4, 4 * 40, dtype=dtype)
        q[0, 0, :40] = 0
        q[0, 1, 40:80] = 0
        q[0, 1, 45] = torch.finfo(F16).max
        q[0, 2, 80:120] = torch.finfo(dtype).smallest_normal
        pos = np.arange(8).reshape(2, 4, 1)
        check_rope(q, None, 40, pos, (24,), eps=1e-6)
        check_rope(q, None, 40, pos, (24,), eps=1e-6, halves=True)
        assert (nv().nv_op_qk_rope(q, None, 40, i32(pos), (24,), nv().nv_rope_freqs((24,)),
                                   eps=1e-6)[0][0, 0, :40] == 0).all()
        was = nv().nv_op_qk_rope(q, None, 40, i32(pos), (24,), nv().nv_rope_freqs((24,)))[0]
        q[1, 1, 41], q[1, 2, 0] = float("nan"), float("inf")
        got = nv().nv_op_qk_rope(q, None, 40, i32(pos), (24,), nv().nv_rope_freqs((24,)))[0]
        assert torch.isnan(got[1, 1, 40:80]).all() and torch.isnan(got[1, 2, 0])
        got[1, 1, 40:80], got[1, 2, :40] = was[1, 1, 40:80], was[1, 2, :40]
        assert torch.equal(got, was)
        plain = nv().nv_op_qk_rope(q, None, 40, i32(pos), (24,), nv().nv_rope_freqs((24,)), eps=None)[0]
        assert torch.isnan(plain[1, 1, 40:80]).sum() <= 2  # only its pair
        q[1, 1, 79] = float("-inf")  # behind the axes: itself
        assert nv().nv_op_qk_rope(q, None, 40, i32(pos), (24,), nv().nv_rope_freqs((24,)),
                                  eps=None)[0][1, 1, 79] == float("-inf")


def test_rope_empty():
    f = nv().nv_rope_freqs((64,))
    q = rand(1, 2, 3, 128, dtype=F16)
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    assert nv().nv_op_qk_rope(q[:, :0], q[:, :0], 64, z(2, 0, 1), (64,), f)[1].shape == (2, 0, 128)
    assert nv().nv_op_qk_rope(q[:0], None, 64, z(0, 3, 1), (64,), f)[0].shape == (0, 3, 128)
    y = nv().nv_op_qk_rope(q, q[:, :, :0], 64, z(2, 3, 1), (64,), f)
    assert y[1].shape == (2, 3, 0) and not torch.isnan(y[0]).any()


# ----------------------------------------------------------------------------- append and read

def pages_np(seed, n, H, dh, lo=118, hi=132):
    """A cache of n pages full of any codes."""
    rng = np.random.default_rng(seed)
    code = lambda: rng.integers(0, 256, (n, H, 64, dh // 2)).astype(np.uint8)
    scale = lambda: rng.integers(lo, hi, (n, H, 64, -(-dh // 32))).astype(np.uint8)
    return [code(), code(), scale(), scale()]


def to_pages(a):
    return tuple(dev(t) for t in a)


def check_append(k, v, pages, table, pos, count, H):
    """k, v device [R][T][H * dh]; pages, table, pos, count NumPy.  All bytes of the cache, and what is
    read of it."""
    R, T, C = k.shape
    d = to_pages(pages)
    cn = None if count is None else i32(count)
    nv().nv_op_kv4_append(k, v, d, i32(table), i32(pos), cn)
    sh = lambda t: np64(t).reshape(R, T, H, C // H)
    ok, oks = O.append(sh(k), pages[0], pages[2], table, pos, count)
    ov, ovs = O.append(sh(v), pages[1], pages[3], table, pos, count)
    got = [t.cpu().numpy() for t in d]
    for g, w, what in zip(got, (ok, ov, oks, ovs), ("kp", "vp", "ks", "vs")):
        assert np.array_equal(g, w), what
    for t in (F32, BF16, F16):
        y = nv().nv_op_kv4_read(d, i32(table), i32(pos), T, cn, t)
        for g, c, s in zip(y, (ok, ov), (oks, ovs)):
            want = torch.from_numpy(O.read(c, s, table, pos, T, count)).to(t)
            assert torch.equal(g.cpu().nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0))
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dh", [16, 32, 40, 64, 80, 128, 160])
@pytest.mark.parametrize("T", [1, 3, 64, 150])
def test_append_and_read(T, dh, dtype):
    print("append4", T, dh, dtype, flush=True)
    R, H, W = 5, 3, 6
    pos = np.array([0, 1, 63, 64, 130])
    k, v = rand(T, R, T, H * dh, dtype=dtype), rand(T + 1, R, T, H * dh, dtype=dtype)
    table = np.random.default_rng(T).permutation(R * W + 2)[:R * W].reshape(R, W).astype(np.int32)
    pages = pages_np(dh, R * W + 2, H, dh)
    check_append(k, v, pages, table, pos, None, H)
    check_append(k, v, pages, table, pos, [T, 0, T // 2 + 1, T + 5, -3], H)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_append_at_the_edges_of_codes_and_scales(dtype):
    """Ties between codes, largest magnitudes next to a scale's limit, every exponent of the type."""
    rng = np.random.default_rng(0)
    ties = np.array([0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, .5, 1, 1.5, 2, 3, 4, 5.75])
    fi = torch.finfo(dtype)
    lo, hi = int(np.log2(fi.smallest_normal)) - (10 if dtype == F16 else 7), int(np.log2(fi.max))
    rows = []
    for p in range(lo - 2, hi + 1):
        for top in (1.0, 1.5, 1.5 + fi.eps * 2, 1.99):
            t = rng.permutation(np.concatenate([ties, -ties])) * 2.0 ** (p - 2) / (1 if top > 1.2 else 2)
            t[np.abs(t) > top * 2.0 ** p] = 0
            t[rng.integers(32)] = top * 2.0 ** p
            rows.append(t)
    with np.errstate(over="ignore"):
        x = torch.from_numpy(np.array(rows)).to(dtype).cuda()[None]
    T = x.shape[1]
    W = -(-T // 64)
    check_append(x, -x, pages_np(1, W, 1, 32), np.arange(W, dtype=np.int32)[None], np.array([0]), None, 1)


def test_append_that_stores_nothing_or_drops():
    """Holes, pages past the pool, negative positions, tokens past the table's end."""
    R, H, dh, T = 6, 1, 40, 100
    pages = pages_np(3, 7, H, dh)
    table = np.array([[-1, 0], [1, 7], [2, 100000], [3, 4], [5, 6], [-5, -1]], np.int32)
    k, v = rand(5, R, T, dh, dtype=BF16), rand(6, R, T, dh, dtype=BF16)
    got = check_append(k, v, pages, table, np.array([10, 10, 10, -1, 120, 0]), None, H)
    for i in (3, 4, 5):  # nothing of row 3; only page 6 of row 4
        assert np.array_equal(got[0][i], pages[0][i])
    big = 2 ** 31 - 50  # positions whose end passes 32 bits
    check_append(k[:1], v[:1], pages, table[:1], np.array([big]), None, H)


def test_append_of_what_is_not_finite_and_of_views():
    """A block with a NaN or an infinity is NaN, its neighbours are not."""
    R, H, dh, T = 2, 2, 128, 70
    qkv = rand(7, R, T, 3 * H * dh + 5, dtype=F16)
    qkv[0, 3, 300], qkv[0, 4, 301], qkv[1, 60, 600] = float("inf"), float("nan"), float("-inf")
    qkv[1, :, 256:384] = 0
    table = np.array([[3, 1, 0], [2, 4, 5]], np.int32)
    pages = pages_np(8, 6, H, dh)
    for a, b in ((256, 512), (3, 259)):  # aligned views of one product's output, and odd ones
        got = check_append(qkv[:, :, a:a + 256], qkv[:, :, b:b + 256], pages, table, np.array([0, 60]),
                           None, H)
        assert (got[2][3] == 255).sum() + (got[3][3] == 255).sum() == 2  # keys, then values
    one = qkv[:, :1, 256:512].expand(R, T, 256)  # a token's stride of zero
    check_append(one, one, pages, table, np.array([5, 1]), [70, 3], H)


def test_tokens_written_in_any_order_and_again():
    """Parts of a prompt last one first, some of it twice: the cache of one call, nothing else touched."""
    R, H, dh, T = 2, 2, 80, 150
    k, v = rand(1, R, T, H * dh, dtype=F16), rand(2, R, T, H * dh, dtype=F16)
    table = i32([[4, 1, 5], [0, 3, 2]])
    one, parts = (to_pages(pages_np(3, 7, H, dh)) for _ in range(2))
    pos = np.array([3, 40])
    nv().nv_op_kv4_append(k, v, one, table, i32(pos))
    for a, b in ((100, 150), (7, 101), (0, 70), (20, 21)):
        nv().nv_op_kv4_append(k[:, a:b], v[:, a:b], parts, table, i32(pos + a))
    for a, b in zip(one, parts):
        assert torch.equal(a, b)


def test_cache_past_32_bits():
    """Pages whose codes lie more than 2^32 bytes into the cache: written, read and attended as the same
    pages of a small cache."""
    H, dh, n = 8, 128, 140_000  # 32 KiB of codes a page: 4.6e9 bytes
    P = nv()
    big = (*(torch.empty(n, H, 64, dh // 2, dtype=torch.uint8, device="cuda") for _ in "kv"),
           *(torch.empty(n, H, 64, dh // 32, dtype=torch.uint8, device="cuda") for _ in "kv"))
    small = P.nv_kv4_pages(6, H, dh, "cuda")
    ids = np.array([[n - 1, 5, n - 2], [131_072, 131_071, n - 3]])
    tb, ts = i32(ids), i32(np.arange(6).reshape(2, 3))
    k, v = rand(1, 2, 190, H * dh, dtype=F16), rand(2, 2, 190, H * dh, dtype=F16)
    pos = i32([0, 0])
    for d, t in ((big, tb), (small, ts)):
        P.nv_op_kv4_append(k, v, d, t, pos)
    for a, b in zip(P.nv_op_kv4_read(big, tb, pos, 190), P.nv_op_kv4_read(small, ts, pos, 190)):
        assert torch.equal(a, b)
    want, _ = O.quantise(np64(k).reshape(2, 190, H, dh))
    assert np.array_equal(big[0][n - 1, :, 7].cpu().numpy(), want[0, 7])
    for S in (1, 300):
        q = rand(3, 2, S, 2 * H * dh, dtype=F16)
        for lens in ([190, 180], [7, 100]):
            assert torch.equal(P.nv_op_attention_kv4(q, big, tb, i32(lens), 0.1),
                               P.nv_op_attention_kv4(q, small, ts, i32(lens), 0.1))


def test_read_into_views_and_of_any_byte():
    """Rows inside a larger buffer, unaligned ones; every code with every scale."""
    pages = pages_np(9, 5, 2, 40)
    pages[0].reshape(-1)[:256] = np.arange(256)
    pages[2][:] = np.arange(pages[2].size).reshape(pages[2].shape) % 256
    table = np.array([[0, 2], [4, -1]], np.int32)
    d = to_pages(pages)
    pos, count = np.array([0, 30]), [128, 77]
    want = [O.read(c, s, table, pos, 128, count) for c, s in ((pages[0], pages[2]), (pages[1], pages[3]))]
    for at, dtype in ((8, F32), (3, F16), (16, BF16), (1, BF16)):
        big = [torch.full((2, 130, 100), 5.0, dtype=dtype, device="cuda") for _ in "kv"]
        nv().nv_op_kv4_read(d, i32(table), i32(pos), 128, i32(count), dtype,
                            out=tuple(b[:, 1:129, at:at + 80] for b in big))
        for b, w in zip(big, want):
            w = torch.from_numpy(w).to(dtype)
            assert torch.equal(b[:, 1:129, at:at + 80].cpu().nan_to_num(7, 8, 9), w.nan_to_num(7, 8, 9))
            assert (b[:, 0] == 5).all() and (b[:, 129] == 5).all()
            assert (b[:, :, :at] == 5).all() and (b[:, :, at + 80:] == 5).all()


# ----------------------------------------------------------------------------- attention_kv4

def check_attention(q, pages, table, lens, scale, H, qpos=None, copies=1, **kw):
    """q device [R][S][Hq * dh]; the rest NumPy.  copies: the rows so many times over."""
    R, S, C = q.shape
    dh = 2 * pages[0].shape[3]
    many = lambda a: i32(np.concatenate([np.asarray(a)] * copies))
    out = nv().nv_op_attention_kv4(q.repeat(copies, 1, 1) if copies > 1 else q, to_pages(pages), many(table),
                                   many(lens), scale, qpos=None if qpos is None else many(qpos), **kw)
    for i in range(1, copies):
        assert np.array_equal(bits(out[:R]), bits(out[i * R:(i + 1) * R])), i
    out = out[:R]
    with np.errstate(invalid="ignore", over="ignore"):
        o, spread, size, most = O.attention(np64(q).reshape(R, S, C // dh, dh), *pages, table, lens,
                                            scale, H, qpos)
    n = table.shape[1] * 64
    got = np64(out).reshape(o.shape)
    used = pages[3][np.unique(table[(table >= 0) & (table < len(pages[0]))])]
    big = 6 * 2.0 ** (int(np.where(used < 255, used, 0).max(initial=0)) - 127.0)
    rel = 2 * (dh * E * size + 8 * E * most + 4 * E) + 2 * u(F16) + n * E
    tol = rel * spread * (1 + u(q.dtype)) + n * 2.0 ** -34 * (big + np.abs(o)) \
        + u(q.dtype) * np.abs(o) + (2.0 ** -25 if q.dtype == F16 else 0)
    assert np.array_equal(np.isnan(got), np.isnan(o))
    with np.errstate(invalid="ignore"):
        bad = np.abs(got - o) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(),
                           float(np.nanmax(np.abs(got - o) / tol)))
    return out


def a_cache(seed, R, W, H, dh, spare=2):
    """Ordinary keys and values in shuffled pages; the pages of no row hold NaN."""
    rng = np.random.default_rng(seed)
    P = R * W + spare
    k, v = (rng.standard_normal((P, H, 64, dh)) * 2.0 ** rng.integers(-3, 3, (P, H, 1, 1)) for _ in "kv")
    (kq, ks), (vq, vs) = O.quantise(k), O.quantise(v)
    table = rng.permutation(P)[:R * W].reshape(R, W).astype(np.int32)
    free = np.setdiff1d(np.arange(P), table)
    ks[free], vs[free] = 255, 255
    return [kq, vq, ks, vs], table


def spoil(pages, table, lens):
    """NaN scales and large codes in the tokens behind each row's last one."""
    for r, n in enumerate(lens):
        for p in range(max(0, int(n)) // 64, table.shape[1]):
            a = max(0, int(n) - p * 64)
            if 0 <= table[r, p] < pages[0].shape[0]:
                for i, to in enumerate((0x77, 0xF7, 255, 255)):
                    pages[i][table[r, p], :, a:] = to


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dh", [16, 32, 40, 64, 80, 128, 160])
@pytest.mark.parametrize("S,H,G,W", [(1, 2, 1, 5), (1, 1, 8, 9), (3, 2, 4, 3), (70, 1, 2, 2)])
def test_attention(S, H, G, W, dh, dtype):
    print("attention_kv4", S, H, G, W, dh, dtype, flush=True)
    R = 4
    pages, table = a_cache(S + dh, R, W, H, dh)
    lens = [W * 64, 1, 64, W * 64 - 37]
    spoil(pages, table, lens)
    q = rand(S, R, S, H * G * dh, dtype=dtype)
    check_attention(q, pages, table, lens, dh ** -0.5, H)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dh", [40, 64, 128])
@pytest.mark.parametrize("S,G", [(1, 4), (5, 1), (64, 2), (130, 4)])
def test_attention_causal(S, G, dh, dtype):
    """Limits before the first token, inside pages, past the end; rows of nothing."""
    print("attention_kv4 causal", S, G, dh, dtype, flush=True)
    R, W, H = 6, 4, 2
    pages, table = a_cache(S + dh, R, W, H, dh)
    lens = [256, 200, 130, 0, 65, 256]
    qpos = [256 - S, 100, -3, 0, 62, -S - 5]
    spoil(pages, table, lens)
    q = rand(S + 1, R, S, H * G * dh, dtype=dtype)
    out = check_attention(q, pages, table, lens, dh ** -0.5, H, qpos)
    assert (out[3] == 0).all() and (out[5] == 0).all()


@pytest.mark.parametrize("R,S,H,G,dh,W", [(1, 1, 1, 1, 64, 300), (2, 1, 2, 8, 128, 70),
                                          (1, 2, 1, 3, 160, 150), (1, 1, 2, 4, 40, 600)])
def test_attention_long(R, S, H, G, dh, W):
    """Sequences shared out over many workgroups, whole and ragged, some shares empty."""
    print("attention_kv4 long", R, S, H, G, dh, W, flush=True)
    pages, table = a_cache(W, R, W, H, dh)
    q = rand(W, R, S, H * G * dh, dtype=BF16)
    for n in (W * 64, W * 64 - 3, 200, 1):
        check_attention(q, pages, table, [n] * R, dh ** -0.5, H)


def test_attention_tall():
    """Many queries of a short cache, and a prompt's chunk: whole tiles of queries."""
    for R, S, H, G, dh, W, causal in ((2, 600, 2, 1, 40, 2, False), (2, 333, 2, 4, 128, 9, True),
                                      (1, 1024, 1, 1, 64, 16, True), (3, 257, 2, 1, 80, 5, False),
                                      (1, 300, 1, 2, 160, 8, True), (2, 200, 1, 1, 16, 4, True)):
        print("attention_kv4 tall", R, S, H, G, dh, W, causal, flush=True)
        pages, table = a_cache(S, R, W, H, dh)
        lens = [W * 64 - 51 * r for r in range(R)]
        spoil(pages, table, lens)
        q = rand(S, R, S, H * G * dh, dtype=F16)
        check_attention(q, pages, table, lens, dh ** -0.5, H,
                        [n - S for n in lens] if causal else None)


@pytest.mark.parametrize("tile,shares", sorted(PLAN_SIZES))
def test_attention_plans(tile, shares):
    """Every tile of queries with every join of shares: rows of differing length, holes, a causal
    limit."""
    for i, (R, S, Hq, H, dh, W) in enumerate(PLAN_SIZES[tile, shares]):
        print("attention_kv4 plan", R, S, Hq, H, dh, W, flush=True)
        pages, table = a_cache(S + W, R, W, H, dh)
        lens = [W * 64 - (W * 23 * r) % (W * 64) for r in range(R)]
        spoil(pages, table, lens)
        if i:
            table[0, W // 2] = -1
        q = rand(S + W, R, S, Hq * dh, dtype=(BF16, F16)[i])
        check_attention(q, pages, table, lens, dh ** -0.5, H, [n - S for n in lens] if i else None)


def test_attention_holes_and_bad_pages():
    R, H, dh, W = 3, 2, 64, 6
    for S in (2, 90, 300):
        pages, table = a_cache(1, R, W, H, dh)
        table[0, 1], table[0, 5], table[1, 0], table[2] = -1, 10 ** 6, -7, -1
        q = rand(1, R, S, 4 * dh, dtype=F16)
        out = check_attention(q, pages, table, [384, 300, 384], dh ** -0.5, H)
        assert (out[2] == 0).all()
        assert (check_attention(q, pages, table, [-5, 0, 384], 0.1, H) == 0).all()
        check_attention(q, pages, table, [10 ** 9, 2 ** 31 - 1, 7], 0.1, H)  # cut to the table
        check_attention(q, pages, table, [384, 300, 384], 0.1, H, [2 ** 31 - 1, 200, -2 ** 31])


# Queries, query heads a head, copies of the rows: tiles of 16 queries (the first four), of 64, of 128.
SIZES = [(1, 1, 1), (9, 1, 1), (1, 4, 1), (40, 1, 1), (300, 1, 1), (70, 4, 1), (120, 4, 96)]


@pytest.mark.parametrize("S,G,N", SIZES)
def test_attention_scales_far_apart(S, G, N):
    """Values and keys past what a float16 operand holds, in any order, one token of them or blocks of a
    token; blocks of zeros."""
    for dtype in (F16, BF16):
        for dh in (64, 128):
            pages, table = a_cache(2, 1, 5, 1, dh)
            rng = np.random.default_rng(S)
            q = rand(3, 1, S, G * dh, dtype=dtype)
            for keys, vals in (((127, 127), (90, 138)), ((127, 127), (1, 120)), ((96, 126), (120, 130)),
                               ((90, 141), (127, 127)), ((127, 128), (20, 160 if dtype == BF16 else 136))):
                print("attention_kv4 scales", S, G, dtype, dh, keys, vals, flush=True)
                for i, (lo, hi) in ((2, keys), (3, vals)):
                    pages[i][:] = np.where(rng.random(pages[i].shape) < 0.02, lo, 126)
                    pages[i][table[0, 1]] = lo
                    pages[i][table[0, 3], :, 20:23] = hi
                    pages[i][table[0, 2], :, 7] = lo
                    pages[i][table[0, 2], :, 8, -1] = hi
                if max(keys) > 130:  # a few large keys, small queries
                    q = rand(3, 1, S, G * dh, dtype=dtype, scale=2.0 ** -12)
                if dtype == F16:  # results within the type
                    pages[1][table[0, 3], :, 20:23] &= 0x99
                for i in (0, 1):
                    pages[i][table[0, 0], :, 40] = 0
                    pages[i + 2][table[0, 0], :, 40] = 1
                check_attention(q, pages, table, [320], dh ** -0.5, 1, copies=N)
                check_attention(q, pages, table, [310], dh ** -0.5, 1, [310 - S], copies=N)


@pytest.mark.parametrize("S,G,N", SIZES)
def test_attention_peaked_and_large_scores(S, G, N):
    """References that move late, scores of hundreds, one key that takes all."""
    for dtype in (F16, BF16):
        pages, table = a_cache(4, 2, 8, 1, 128)
        pages[2][table[0, 5]] += 4
        pages[2][table[1, 7], :, 3] += 9
        q = rand(5, 2, S, G * 128, dtype=dtype)
        for lens, scale in (([512, 512], 0.1), ([512, 449], -0.1), ([512, 449], 0.0)):
            check_attention(q, pages, table, lens, scale, 1, copies=N)


@pytest.mark.parametrize("S,G,N", SIZES)
@pytest.mark.parametrize("dh", [64, 128])
def test_attention_queries_of_unlike_channels(S, G, N, dh):
    """One channel of some queries far above the others, on keys that are zero there and on some that are
    not; queries of the type's smallest numbers, of one channel alone, of zeros."""
    for dtype in (F16, BF16):
        for far in (100.0, 3000.0, 50000.0):
            pages, table = a_cache(4, 1, 4, 1, dh)
            values = O.values(pages[0], pages[2])
            values[..., 5] = np.where(np.arange(64) % 16 == 3, 2.0 ** -10, 0)
            pages[0], pages[2] = O.quantise(values)
            q = rand(5, 1, S, G * dh, dtype=dtype)
            q[0, ::2, 5] = far
            q[0, 1::3, dh - 1] = 0
            q[0, 2::5, :32] *= 2.0 ** -12
            q[0, 3::7, 1:] = 0
            q[0, 4::7] = torch.finfo(dtype).tiny
            q[0, 5::7] = 0
            check_attention(q, pages, table, [256], dh ** -0.5, 1, copies=N)
            check_attention(q, pages, table, [250], dh ** -0.5, 1, [250 - S], copies=N)
        q[0, S // 2, 7], q[0, 0, 9] = float("inf"), float("nan")
        out = nv().nv_op_attention_kv4(q, to_pages(pages), i32(table), i32([250]), dh ** -0.5)
        assert torch.isnan(out[0, S // 2, :dh]).all() and torch.isnan(out[0, 0, :dh]).all()
        assert torch.isnan(out).sum() == (2 if S > 1 else 1) * dh


@pytest.mark.parametrize("S,G,N", SIZES)
def test_attention_nan_reaches_only_who_sees_it(S, G, N):
    """NaN blocks of keys and values before some query's limit and behind another's."""
    for dtype in (F16, BF16):
        pages, table = a_cache(6, 1, 4, 1, 64)
        q = rand(7, 1, S, G * 64, dtype=dtype)
        first = 250 - S
        at = 250 - (S + 1) // 2
        page = table[0, at // 64]
        pages[3][page, 0, at % 64, 1] = 255
        out = check_attention(q, pages, table, [251], 0.125, 1, [first], copies=N)
        if S > 1:
            assert torch.isnan(out).any() and not torch.isnan(out[0, :S // 2 - 1]).any()
            assert not torch.isnan(out.view(1, S, G, 64)[..., :32]).any()
        pages[2][page, 0, at % 64, 0] = 255
        check_attention(q, pages, table, [251], 0.125, 1, [first], copies=N)
        check_attention(q, pages, table, [at], 0.125, 1, copies=N)  # nobody sees it
        for i in (2, 3):
            pages, table = a_cache(6, 1, 4, 1, 64)
            pages[i][table[0, 3]] = 255
            pages[i][table[0, 0], :, 9] = 255
            check_attention(q, pages, table, [251], 0.125, 1, [first], copies=N)
            check_attention(q, pages, table, [192], 0.125, 1, copies=N)
            check_attention(q, pages, table, [192], 0.125, 1, [9 - S], copies=N)


def test_attention_strides():
    R, S, H, dh = 2, 5, 2, 64
    pages, table = a_cache(8, R, 3, H, dh)
    big = rand(9, R, S, 3 * 256, dtype=F16)
    out = torch.full((R, S + 1, 512), 5.0, dtype=F16, device="cuda")
    check_attention(big[:, :, 256:512], pages, table, [100, 192], 0.125, H, out=out[:, :S, 128:384])
    assert (out[:, S] == 5).all() and (out[:, :, :128] == 5).all() and (out[:, :, 384:] == 5).all()
    q = big[:, :, :256].contiguous()
    x = check_attention(q[:1].expand(2, S, 256), pages, table, [100, 100], 0.125, H)
    assert x.shape == (2, S, 256)


def test_cache_and_attention_empty():
    pages = nv().nv_kv4_pages(3, 2, 64, "cuda")
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    q = rand(0, 2, 3, 128, dtype=F16)
    assert (nv().nv_op_attention_kv4(q, pages, z(2, 0), z(2), 0.1) == 0).all()
    assert nv().nv_op_attention_kv4(q[:, :0], pages, z(2, 1), z(2), 0.1).shape == (2, 0, 128)
    assert nv().nv_op_attention_kv4(q[:0], pages, z(0, 1), z(0), 0.1).shape == (0, 3, 128)
    nv().nv_op_kv4_append(q[:, :0], q[:, :0], pages, z(2, 1), z(2))
    nv().nv_op_kv4_append(q[:0], q[:0], pages, z(0, 1), z(0))
    nv().nv_op_kv4_append(q, q, pages, z(2, 0), z(2))
    assert (nv().nv_op_kv4_read(pages, z(2, 0), z(2), 3)[0] == 0).all()
    assert nv().nv_op_kv4_read(pages, z(2, 1), z(2), 0)[0].shape == (2, 0, 128)
    assert nv().nv_op_kv4_read(pages, z(0, 1), z(0), 3)[1].shape == (0, 3, 128)


# ---------------------------------------------------------------------------------- together

class Layer:
    """norm -> q|k|v -> norm of heads and rotation -> append -> attention -> output product + residual
    -> norm, on a 4-bit cache."""

    def __init__(self, R, D, Hq, H, dh, W, dtype):
        self.Hq, self.H, self.dh, self.dtype = Hq, H, dh, dtype
        P = nv()
        self.w1, self.w2 = 1 + 0.1 * rand(1, D), 1 + 0.1 * rand(2, D)
        self.wq, self.wk = 1 + 0.1 * rand(6, dh), 1 + 0.1 * rand(7, dh)
        self.wqkv = P.nv_op_quant8(rand(3, (Hq + 2 * H) * dh, D, scale=D ** -0.5), block_rows=128)
        self.wo = P.nv_op_quant8(rand(4, D, Hq * dh, scale=(Hq * dh) ** -0.5), block_rows=128)
        self.pages = P.nv_kv4_pages(R * W, H, dh, "cuda")
        self.axes = (dh // 4, dh // 2)
        self.freqs = P.nv_rope_freqs(self.axes)
        self.table = torch.randperm(R * W, generator=torch.Generator().manual_seed(5)).view(
            R, W).int().cuda()

    def __call__(self, x, r, pos, count):
        """x, r [R * T][D]; returns (qkv, q, k, attention, codes, scales, h) of the next norm."""
        P, R = nv(), self.table.shape[0]
        C, Ck = self.Hq * self.dh, self.H * self.dh
        q, s, h = P.nv_op_rmsnorm8(x, self.w1, residual=r)
        qkv = P.nv_op_linear8(q, s, *self.wqkv, dtype=self.dtype).view(R, -1, C + 2 * Ck)
        at = pos[:, None] + torch.arange(qkv.shape[1], device="cuda", dtype=torch.int32)
        places = torch.stack((at // 8, at % 8), -1)  # rows and columns of a grid
        q, k = P.nv_op_qk_rope(qkv[:, :, :C], qkv[:, :, C:C + Ck], self.dh, places, self.axes, self.freqs,
                               self.wq, self.wk)
        P.nv_op_kv4_append(k, qkv[:, :, C + Ck:], self.pages, self.table, pos, count)
        a = P.nv_op_attention_kv4(q, self.pages, self.table, pos + count, self.dh ** -0.5, qpos=pos)
        aq, as_ = P.nv_op_quant8(a.reshape(-1, C))
        y = P.nv_op_linear8(aq, as_, *self.wo, residual=h, dtype=self.dtype)
        return (qkv, q, k, a) + P.nv_op_rmsnorm8(y, self.w2, residual=h)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_layer_of_all_of_them(dtype):
    """A prompt, then single tokens, each step held to the oracle on that step's own inputs."""
    R, T, D, Hq, H, dh, W = 3, 100, 640, 10, 2, 64, 4
    layer = Layer(R, D, Hq, H, dh, W, dtype)
    pos = torch.zeros(R, dtype=torch.int32, device="cuda")
    C, Ck = Hq * dh, H * dh
    for step, count in enumerate(([100, 37, 64], [1, 1, 1], [1, 0, 1], [1, 1, 1])):
        n = T if step == 0 else 1
        count = torch.tensor(count, dtype=torch.int32, device="cuda")
        x, r = rand(10 + step, R * n, D, dtype=dtype), rand(20 + step, R * n, D, dtype=dtype)
        was = [bits(t) for t in layer.pages]
        qkv, q, k, a, q2, s2, h2 = layer(x, r, pos, count)
        tb, ps, cn = layer.table.cpu().numpy(), pos.cpu().numpy(), count.cpu().numpy()
        at = ps[:, None] + np.arange(n)
        check_rope(qkv[:, :, :C], qkv[:, :, C:C + Ck], dh, np.stack((at // 8, at % 8), -1), layer.axes,
                   layer.wq, layer.wk)
        sh = lambda t: np64(t).reshape(R, n, H, dh)
        ok, oks = O.append(sh(k), was[0], was[2], tb, ps, cn)
        ov, ovs = O.append(sh(qkv[:, :, C + Ck:]), was[1], was[3], tb, ps, cn)
        for g, w in zip(layer.pages, (ok, ov, oks, ovs)):
            assert np.array_equal(bits(g), w)
        check_attention(q, [ok, ov, oks, ovs], tb, ps + cn, dh ** -0.5, H, ps)
        got = nv().nv_op_kv4_read(layer.pages, layer.table, pos * 0, 256, pos + count, dtype)
        want = O.read(ok, oks, tb, ps * 0, 256, ps + cn)
        assert np.array_equal(np64(got[0]), want)
        o = nv().nv_op_attention_kv4(q, layer.pages, layer.table, pos + count, dh ** -0.5, qpos=pos)
        assert torch.equal(o, a)
        assert not torch.isnan(h2).any() and not ((bits(q2) & 127) == 127).any()
        pos = pos + count


def test_layer_on_another_stream_and_in_a_graph():
    """Single-token steps captured once and replayed: every replay equals the eager step."""
    R, D, Hq, H, dh, W = 4, 640, 8, 2, 128, 40
    eager, graph = (Layer(R, D, Hq, H, dh, W, F16) for _ in range(2))
    fill = torch.tensor([2400, 5, 64, 700], dtype=torch.int32, device="cuda")
    for layer in (eager, graph):  # a prompt's keys and values
        k, v = rand(1, R, 2400, H * dh, dtype=F16), rand(2, R, 2400, H * dh, dtype=F16)
        nv().nv_op_kv4_append(k, v, layer.pages, layer.table, fill * 0, fill)
    x, r = rand(3, R, D, dtype=F16), rand(4, R, D, dtype=F16)
    pos, one = fill.clone(), torch.ones_like(fill)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # the first token, on a stream of its own
        want0 = [t.clone() for t in eager(x, r, pos, one)]
        got0 = [t.clone() for t in graph(x, r, pos, one)]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(want0, got0):
        assert np.array_equal(bits(a), bits(b))
    g = torch.cuda.CUDAGraph()
    pos += 1
    with torch.cuda.graph(g):
        outs = graph(x, r, pos, one)
    for step in range(4):
        x.copy_(rand(30 + step, R, D, dtype=F16))
        r.copy_(rand(40 + step, R, D, dtype=F16))
        torch.cuda.synchronize()
        g.replay()
        want = eager(x, r, pos, one)
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert np.array_equal(bits(a), bits(b)), step
        for a, b in zip(eager.pages, graph.pages):
            assert np.array_equal(bits(a), bits(b)), step
        pos += 1


def test_calls_repeat_to_the_bit():
    """No order of atomics: the same call gives the same bits, also beside another stream's."""
    P = nv()
    pages, table = a_cache(9, 2, 100, 2, 128)
    d, tb, lens = to_pages(pages), i32(table), i32([6400, 3001])
    q, many = rand(1, 2, 1, 8 * 128, dtype=F16), rand(2, 2, 300, 8 * 128, dtype=BF16)
    f = P.nv_rope_freqs((128,))
    places = i32(np.arange(600).reshape(2, 300, 1))

    def all_of_them():
        return (P.nv_op_attention_kv4(q, d, tb, lens, 0.1), P.nv_op_attention_kv4(many, d, tb, lens, 0.1),
                *P.nv_op_qk_rope(many, many[:, :, :256], 128, places, (128,), f, halves=True),
                *P.nv_op_kv4_read(d, tb, lens * 0, 300, None, F16))
    first = all_of_them()
    torch.cuda.synchronize()
    got = []
    for s in (torch.cuda.Stream(), torch.cuda.Stream()) * 3:
        with torch.cuda.stream(s):
            got.append(all_of_them())
    torch.cuda.synchronize()
    for g in got:
        for a, b in zip(first, g):
            assert torch.equal(a, b)


def test_two_graphs_with_workspaces_of_their_own():
    """Captured calls that share nothing but the cache, replayed in turn and with eager calls between."""
    P = nv()
    pages, table = a_cache(9, 2, 100, 2, 64)
    d, tb, lens = to_pages(pages), i32(table), i32([6400, 3001])
    qs = [rand(i, 2, 1, 8 * 64, dtype=BF16) for i in range(2)]
    graphs, outs = [], []
    P.nv_op_attention_kv4(qs[0], d, tb, lens, 0.1)
    torch.cuda.synchronize()
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(P.nv_op_attention_kv4(q, d, tb, lens, 0.1))
        graphs.append(g)
    for step in range(3):
        for i, q in enumerate(qs):
            q.copy_(rand(10 * step + i, 2, 1, 8 * 64, dtype=BF16))
        for g in graphs:
            g.replay()
        want = [P.nv_op_attention_kv4(q, d, tb, lens, 0.1) for q in qs]
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), step
