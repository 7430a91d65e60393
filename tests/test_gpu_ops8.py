"""The 8-bit operators against their float64 oracle.

Bounds.  u(t) = torch.finfo(t).eps / 2 is one rounding to t, E = 2^-23 one float32 operation (a
whole step: the matrix unit's own rounding of its sums is not specified to be to nearest).
  codes       scaling by a power of two is exact, so codes and scales are the oracle's to the bit
  norm        the sum of squares passes at most 32 + 6 + 16 float32 additions (a thread's values in
              turn, a wave's tree, the waves): 54 E, halved by the root, and some ten operations
              around it: 40 E of a value before its code is chosen; then half a code's step
  product     The e4m3 matrix unit adds products in groups of eight consecutive k, and cuts each to
              2^-13 of 2^(largest exponent of the group) first, towards zero (seen with one large
              product and a small one: lost below 2^-13 of it within its group of eight, kept to
              2^-23 outside).  The largest loses nothing, the other seven less than 2^-13 of it
              each, and it is at most max |x| max |w| of the group: 7 * 2^-13 of the product of the
              groups' maxima.  Then K float32 additions: K E of sum |x w|; bias and residual 2 E of
              their sizes, one rounding u(t)
  attention   a score is dh float32 additions and three products: (dh E sum |q k| + 4 E |score|)
              absolute, the shift by the maximum and the exponential 4 E |score| + 4 E; twice that
              (numerator and sum) is a probability's relative error; its rounding to float16 is
              2^-11 relative, in numerator and sum, or 2^-25 absolute where it is subnormal (the
              reference maximum is at most the true one); sums of n terms in float32: n E; all of
              sum p |v|, and one rounding u(t) of the result
"""
import numpy as np
import pytest
import torch

from oracle import ops8 as O
from ops8_sizes import FORM_SIZES, PLAN_SIZES

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


def codes_of(a):
    """NumPy codes as a device e4m3 matrix in rows of a multiple of 16 bytes."""
    M, K = a.shape
    t = torch.full((M, -(-K // 16) * 16), 0x7F, dtype=torch.uint8)  # NaN behind the rows
    t[:, :K] = torch.from_numpy(a)
    return t.cuda().view(torch.float8_e4m3fn)[:, :K]


def bytes_of(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def nv():
    import paper_2312_04429_amd as P
    return P


# ------------------------------------------------------------------------------------ quant8

@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 128), (3, 200), (130, 129), (257, 72), (128, 640),
                                 (5, 1000), (300, 1280)])
def test_quant8_codes(M, K, dtype, rows):
    print("quant8", M, K, dtype, rows, flush=True)
    x = rand(M + K, M, K, dtype=F32) * torch.exp2(torch.randint(-12, 12, (M, 1)).float()).cuda()
    x[0, 0] = 0
    x = x.to(dtype)
    q, s = nv().nv_op_quant8(x, block_rows=rows)
    oq, os_ = O.quantise(np64(x), rows)
    assert np.array_equal(bits(s), os_)
    assert np.array_equal(bits(q), oq)
    for t in (F32, BF16, F16):
        y = nv().nv_op_dequant8(q, s, block_rows=rows, dtype=t)
        want = torch.from_numpy(O.values(oq, os_, rows)).to(t)
        assert torch.equal(y.cpu(), want)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_quant8_of_what_is_not_ordinary(dtype, rows):
    """Zero blocks, infinities, NaN, the type's largest and smallest values, block edges."""
    x = rand(1, 200, 300, dtype=dtype)
    fi = torch.finfo(dtype)
    x[0, :] = 0
    x[1, 5], x[1, 140], x[2, 200], x[3, 0] = float("inf"), float("-inf"), float("nan"), fi.max
    x[4, 256:] = float("nan")
    x[5, :] = fi.tiny
    x[6, 128:256] = fi.smallest_normal / 4
    x[130:, 128:] = 0
    q, s = nv().nv_op_quant8(x, block_rows=rows)
    oq, os_ = O.quantise(np64(x), rows)
    assert np.array_equal(bits(s), os_)
    got = bits(q)
    nan = (oq & 127) == 127
    assert np.array_equal((got & 127) == 127, nan)
    assert np.array_equal(got[~nan], oq[~nan])


def test_quant8_strided_and_unaligned():
    """Rows that start anywhere: a column slice at an odd offset, and padded rows."""
    base = rand(2, 37, 523, dtype=BF16)
    for x in (base[:, 3:], base[:, 8:520], base[::3, 1:130]):
        q, s = nv().nv_op_quant8(x)
        oq, os_ = O.quantise(np64(x))
        assert np.array_equal(bits(q), oq) and np.array_equal(bits(s), os_)
        y = nv().nv_op_dequant8(q, s, dtype=BF16)
        assert torch.equal(y.cpu(), torch.from_numpy(O.values(oq, os_)).to(BF16))


def test_quant8_empty():
    q, s = nv().nv_op_quant8(torch.empty(0, 200, dtype=F16, device="cuda"))
    assert q.shape == (0, 200) and s.shape == (0, 2)
    assert nv().nv_op_dequant8(q, s).shape == (0, 200)


# ---------------------------------------------------------------------------------- rmsnorm8

def check_norm(x, w, r, eps=1e-6):
    q, s, h = nv().nv_op_rmsnorm8(x, w, residual=r, eps=eps)
    if r is None:
        assert h is None
    else:  # float32 sum, rounded once: the same in torch
        assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
    y = O.rmsnorm(np64(x), np64(w), None if r is None else np64(r), eps)
    d = 40 * E
    M, D = y.shape
    sb = bits(s)
    for j in range(0, D, 128):
        top = np.abs(y[:, j:j + 128]).max(1)
        lo, hi = O.scale_byte(top * (1 - d)), O.scale_byte(top * (1 + d))
        assert ((sb[:, j // 128] == lo) | (sb[:, j // 128] == hi)).all()
    f = np.repeat(O.scale_value(sb), 128, 1)[:, :D]
    got = O.VALUES[bits(q)] * f
    # a code's half step: 2^-4 of the value, 2^-10 of the scale below its smallest normal number
    half = np.maximum(np.abs(y) * 2.0 ** -4, f * 2.0 ** -10)
    assert (np.abs(got - y) <= half * (1 + d) + d * np.abs(y)).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,D", [(1, 1), (3, 64), (5, 200), (130, 129), (7, 513), (64, 1280),
                                 (9, 1025), (33, 2048), (5, 2049), (4, 4096), (3, 5000), (2, 8192),
                                 (2, 8200), (1, 20001), (2, 32768)])
def test_rmsnorm8(M, D, dtype):
    print("rmsnorm8", M, D, dtype, flush=True)
    x, r = rand(M, M, D, dtype=dtype), rand(D, M, D, dtype=dtype, scale=3.0)
    w = 1 + 0.2 * rand(7, D)
    check_norm(x, w, r)
    check_norm(x, w, None)


def test_rmsnorm8_strides_and_sizes_of_values():
    base = rand(3, 9, 1500, dtype=F16)
    check_norm(base[:, 5:1005], 1 + 0.1 * rand(4, 1000), base[:, 300:1300])
    check_norm(base[:, 8:1288], 1 + 0.1 * rand(4, 1280), None)
    x = rand(5, 6, 512, dtype=BF16) * torch.tensor([1e-20, 1e-3, 1.0, 1e3, 1e15, 0.0]).cuda()[:, None]
    check_norm(x.to(BF16), 1 + 0.1 * rand(6, 512), None)


def test_rmsnorm8_in_place_at_the_c_entry():
    """h may be the residual itself."""
    from paper_2312_04429_amd import _native as N
    from paper_2312_04429_amd.api import _p, _stream
    x, r, w = rand(8, 20, 1280, dtype=F16), rand(9, 20, 1280, dtype=F16), 1 + 0.1 * rand(10, 1280)
    q, s, h = nv().nv_op_rmsnorm8(x, w, residual=r)
    r2, q2, s2 = r.clone(), torch.empty_like(q), torch.empty_like(s)
    N.check(N.lib.nv_op_rmsnorm8(_p(x), 1280, _p(r2), 1280, N.NV_F16, _p(w), 1e-6, 20, 1280, _p(r2),
                                 1280, _p(q2), q2.stride(0), _p(s2), _stream()), "nv_op_rmsnorm8")
    assert torch.equal(r2, h) and np.array_equal(bits(q2), bits(q)) and np.array_equal(bits(s2), bits(s))


def test_rmsnorm8_row_that_is_not_finite():
    x = rand(11, 3, 256, dtype=F16)
    x[1, 7] = float("nan")
    q, s, _ = nv().nv_op_rmsnorm8(x, torch.ones(256, device="cuda"))
    assert ((bits(q)[1] & 127) == 127).all()
    assert not ((bits(q)[[0, 2]] & 127) == 127).any()


# ----------------------------------------------------------------------------------- linear8

def check_linear(M, N, K, dtype, bias=True, res=True, seed=0, xexp=None, **kw):
    print("linear8", M, N, K, dtype, bias, res, flush=True)
    rng = np.random.default_rng(seed + M + N + K)
    xq, xs = O.quantise(rng.standard_normal((M, K)) * (2.0 ** rng.integers(-6, 7, (M, 1))))
    wq, ws = O.quantise(rng.standard_normal((N, K)) * 0.02, 128)
    if xexp is not None:
        xs = xexp(xs)
    b = rand(seed + 1, N) if bias else None
    r = rand(seed + 2, M, N, dtype=dtype) if res else None
    out = nv().nv_op_linear8(codes_of(xq), bytes_of(xs), codes_of(wq), bytes_of(ws), bias=b,
                             residual=r, dtype=dtype, **kw)
    xv, wv = (torch.from_numpy(t).cuda() for t in (O.values(xq, xs), O.values(wq, ws, 128)))
    y, size = xv @ wv.T, xv.abs() @ wv.abs().T
    tops = [torch.nn.functional.pad(t.abs(), (0, -K % 8)).view(t.shape[0], -1, 8).amax(2)
            for t in (xv, wv)]
    tol = K * E * size + 7 * 2.0 ** -13 * (tops[0] @ tops[1].T)
    for t in (b, r):
        if t is not None:
            y, tol = y + t.double(), tol + 2 * E * (t.double().abs() + size)
    tol = tol * (1 + u(dtype)) + u(dtype) * y.abs()
    bad = (out.double() - y).abs() > tol
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(),
                           float(((out.double() - y).abs() / tol).max()))
    return out


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 16), (2, 17, 33), (1, 1280, 5120),
                                   (8, 640, 1024), (15, 130, 200), (16, 128, 128), (17, 129, 127),
                                   (33, 257, 384), (64, 320, 1000), (65, 1000, 1280),
                                   (127, 640, 640), (200, 333, 517), (300, 1280, 2000),
                                   (513, 640, 320), (1000, 2560, 640), (2100, 1300, 1290)])
def test_linear8(M, N, K, dtype):
    check_linear(M, N, K, dtype)


@pytest.mark.parametrize("form", sorted(FORM_SIZES))
def test_linear8_forms(form):
    for i, s in enumerate(FORM_SIZES[form]):
        check_linear(*s, (F16, BF16)[i % 2], bias=i % 2 == 0, res=i % 3 != 1)


@pytest.mark.parametrize("bias,res", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("M,N,K", [(3, 200, 2000), (96, 640, 4096), (700, 640, 640)])
def test_linear8_epilogues(M, N, K, bias, res):
    check_linear(M, N, K, BF16, bias, res)


@pytest.mark.parametrize("M", [3, 70, 300])
def test_linear8_scales_over_their_range(M):
    """Scale bytes of differing size in one row, some blocks far below others."""
    spread = lambda s: (s.astype(int) + np.random.default_rng(5).integers(-20, 20, s.shape)).astype(np.uint8)
    check_linear(M, 257, 1100, BF16, xexp=spread)


def test_linear8_long_k():
    """More 128-deep tiles than the scales of one stage."""
    check_linear(200, 300, 40 * 128 + 8, F16)
    check_linear(5, 140, 20000, BF16)


def test_linear8_strides():
    M, N, K = 40, 200, 4096
    big = torch.full((M, N + 8), 7.0, dtype=F16, device="cuda")
    out = check_linear(M, N, K, F16, out=big[:, 4:4 + N])
    assert out.data_ptr() == big.data_ptr() + 8
    assert (big[:, :4] == 7).all() and (big[:, 4 + N:] == 7).all()
    big = torch.full((M, N + 7), 7.0, dtype=F16, device="cuda")  # rows that no vector store fits
    check_linear(M, N, K, F16, out=big[:, 3:3 + N])
    assert (big[:, :3] == 7).all() and (big[:, 3 + N:] == 7).all()


@pytest.mark.parametrize("M,N,K", [(5, 200, 300), (90, 333, 640), (700, 640, 256), (4100, 4200, 300)])
def test_linear8_residual_is_the_output(M, N, K):
    """The sum into the residual's own memory: the bits of the call that writes elsewhere."""
    q, s = nv().nv_op_quant8(rand(0, M, K))
    w, ws = nv().nv_op_quant8(rand(1, N, K), block_rows=128)
    r = rand(2, M, N, dtype=BF16)
    want = nv().nv_op_linear8(q, s, w, ws, residual=r, dtype=BF16)
    got = r.clone()
    assert nv().nv_op_linear8(q, s, w, ws, residual=got, dtype=BF16, out=got) is got
    assert torch.equal(got, want) and not torch.isnan(got).any()


def test_linear8_nan_stays_in_its_row_and_column():
    xq, xs = O.quantise(np.random.default_rng(0).standard_normal((70, 300)))
    wq, ws = O.quantise(np.random.default_rng(1).standard_normal((150, 300)), 128)
    xq[3, 299], wq[140, 0] = 0x7F, 0xFF
    for rows in (slice(0, 70), slice(0, 5)):
        out = nv().nv_op_linear8(codes_of(xq[rows]), bytes_of(xs[rows]), codes_of(wq), bytes_of(ws))
        nan = torch.isnan(out).cpu().numpy()
        want = np.zeros_like(nan)
        want[3, :] = want[:, 140] = True
        assert np.array_equal(nan, want)


def test_linear8_empty():
    q, s = nv().nv_op_quant8(torch.empty(0, 256, dtype=F16, device="cuda"))
    w, ws = nv().nv_op_quant8(rand(0, 64, 256), block_rows=128)
    assert nv().nv_op_linear8(q, s, w, ws).shape == (0, 64)


# -------------------------------------------------------------------------------- kv8 append

def pages_np(seed, n, H, dh, lo=110, hi=125):
    """A cache of n pages full of ordinary codes."""
    rng = np.random.default_rng(seed)
    code = lambda *sh: (rng.integers(0, 119, sh) | (rng.integers(0, 2, sh) << 7)).astype(np.uint8)
    return [code(n, H, 64, dh), code(n, H, dh, 64), rng.integers(lo, hi, (n, H)).astype(np.uint8),
            rng.integers(lo, hi, (n, H)).astype(np.uint8)]


def to_pages(a):
    return tuple(bytes_of(t) for t in a)


def check_append(k, v, pages, table, pos, count, H):
    """k, v device [R][T][H * dh]; pages, table, pos, count NumPy."""
    R, T, C = k.shape
    dev = to_pages(pages)
    i32 = lambda a: bytes_of(np.asarray(a, np.int32))
    nv().nv_op_kv8_append(k, v, dev, i32(table), i32(pos), None if count is None else i32(count))
    cnt = np.full(R, T) if count is None else np.asarray(count)
    sh = lambda t: np64(t).reshape(R, T, H, C // H)
    ok, oks = O.append(sh(k), pages[0], pages[2], table, pos, cnt, False)
    ov, ovs = O.append(sh(v), pages[1], pages[3], table, pos, cnt, True)
    got = [t.cpu().numpy() for t in dev]
    for g, w, what in zip(got, (ok, ov, oks, ovs), ("kp", "vp", "ks", "vs")):
        if what in ("kp", "vp"):
            nan = (w & 127) == 127
            assert np.array_equal((g & 127) == 127, nan), what
            g, w = np.where(nan, 0, g), np.where(nan, 0, w)
        assert np.array_equal(g, w), what
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dh", [16, 32, 40, 64, 80, 128, 160])
@pytest.mark.parametrize("T", [1, 3, 64, 150])
def test_append(T, dh, dtype):
    print("append", T, dh, dtype, flush=True)
    R, H, W = 5, 3, 6
    pos = np.array([0, 1, 63, 64, 130])
    k, v = rand(T, R, T, H * dh, dtype=dtype), rand(T + 1, R, T, H * dh, dtype=dtype)
    table = np.random.default_rng(T).permutation(R * W + 2)[:R * W].reshape(R, W).astype(np.int32)
    pages = pages_np(dh, R * W + 2, H, dh)
    check_append(k, v, pages, table, pos, None, H)
    check_append(k, v, pages, table, pos, [T, 0, T // 2 + 1, T + 5, -3], H)


@pytest.mark.parametrize("T", [2, 5, 40])
def test_append_scales_grow_and_stay(T):
    """Old scales above, at and below what the new tokens need, old codes that become subnormal."""
    R, H, dh = 4, 2, 64
    for old in (90, 115, 118, 119, 120, 140, 254):
        pages = pages_np(old, R * 2, H, dh, old, old + 1)
        table = np.arange(R * 2, dtype=np.int32).reshape(R, 2)
        k, v = rand(1, R, T, H * dh, dtype=F16), rand(2, R, T, H * dh, dtype=F16, scale=4.0)
        check_append(k, v, pages, table, np.array([5, 63, 64, 70]), None, H)


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
    R, H, dh, T = 2, 2, 128, 70
    qkv = rand(7, R, T, 3 * H * dh + 5, dtype=F16)
    qkv[0, 3, 300], qkv[0, 4, 301], qkv[1, 60, 600] = float("inf"), float("nan"), float("-inf")
    qkv[1, :, 256:384] = 0
    table = np.array([[3, 1, 0], [2, 4, 5]], np.int32)
    pages = pages_np(8, 6, H, dh)
    for a, b in ((256, 512), (3, 259)):  # aligned views of one product's output, and odd ones
        check_append(qkv[:, :, a:a + 256], qkv[:, :, b:b + 256], pages, table, np.array([0, 60]),
                     None, H)


# ----------------------------------------------------------------------------- attention_kv8

def check_attention(q, pages, table, lens, scale, H, qpos=None, **kw):
    """q device [R][S][Hq * dh]; the rest NumPy."""
    R, S, C = q.shape
    dh = pages[0].shape[3]
    i32 = lambda a: bytes_of(np.asarray(a, np.int32))
    out = nv().nv_op_attention_kv8(q, to_pages(pages), i32(table), i32(lens), scale,
                                   qpos=None if qpos is None else i32(qpos), **kw)
    with np.errstate(invalid="ignore", over="ignore"):
        o, spread, size, most = O.attention(np64(q).reshape(R, S, C // dh, dh), *pages, table, lens,
                                            scale, H, qpos)
    n = table.shape[1] * 64
    got = np64(out).reshape(o.shape)
    big = np.nanmax(np.abs(O.VALUES[pages[1]]), initial=0) * \
        2.0 ** (int(np.where(pages[3] < 255, pages[3], 0).max()) - 127.0)
    rel = 2 * (dh * E * size + 8 * E * most + 4 * E) + 2 * u(F16) + n * E
    tol = rel * spread * (1 + u(q.dtype)) + n * 2.0 ** -25 * (big + np.abs(o)) \
        + u(q.dtype) * np.abs(o) + (2.0 ** -25 if q.dtype == F16 else 0)
    assert np.array_equal(np.isnan(got), np.isnan(o))
    with np.errstate(invalid="ignore"):
        bad = np.abs(got - o) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(),
                           float(np.nanmax(np.abs(got - o) / tol)))
    return out


def a_cache(seed, R, W, H, dh, spare=2):
    """Codes of unit-sized keys and values in shuffled pages; NaN in the pages nobody names."""
    rng = np.random.default_rng(seed)
    P = R * W + spare
    k, v = rng.standard_normal((P, H, 64, dh)), rng.standard_normal((P, H, dh, 64))
    kq, vq = np.empty(k.shape, np.uint8), np.empty(v.shape, np.uint8)
    ks, vs = np.empty((P, H), np.uint8), np.empty((P, H), np.uint8)
    for a, q, s in ((k, kq, ks), (v, vq, vs)):
        f = 2.0 ** rng.integers(-3, 3, (P, H, 1, 1))
        s[:] = O.scale_byte(np.abs(a * f).max((2, 3)))
        q[:] = O.encode(a * f / O.scale_value(s)[..., None, None])
    table = rng.permutation(P)[:R * W].reshape(R, W).astype(np.int32)
    free = np.setdiff1d(np.arange(P), table)
    kq[free], vq[free] = 0x7F, 0xFF
    return [kq, vq, ks, vs], table


def spoil(pages, table, lens):
    """NaN codes in the tokens behind each row's last one."""
    for r, n in enumerate(lens):
        for p in range(max(0, int(n)) // 64, table.shape[1]):
            a = max(0, int(n) - p * 64)
            if 0 <= table[r, p] < pages[0].shape[0]:
                pages[0][table[r, p], :, a:] = 0x7F
                pages[1][table[r, p], :, :, a:] = 0xFF


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dh", [16, 32, 40, 64, 80, 128, 160])
@pytest.mark.parametrize("S,H,G,W", [(1, 2, 1, 5), (1, 1, 8, 9), (3, 2, 4, 3), (70, 1, 2, 2)])
def test_attention(S, H, G, W, dh, dtype):
    print("attention_kv8", S, H, G, W, dh, dtype, flush=True)
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
    print("attention_kv8 causal", S, G, dh, dtype, flush=True)
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
    print("attention_kv8 long", R, S, H, G, dh, W, flush=True)
    pages, table = a_cache(W, R, W, H, dh)
    q = rand(W, R, S, H * G * dh, dtype=BF16)
    for n in (W * 64, W * 64 - 3, 200, 1):
        check_attention(q, pages, table, [n] * R, dh ** -0.5, H)


def test_attention_tall():
    """Many queries of a short cache, and a prompt's chunk: whole tiles of queries."""
    for R, S, H, G, dh, W, causal in ((2, 600, 2, 1, 40, 2, False), (2, 333, 2, 4, 128, 9, True),
                                      (1, 1024, 1, 1, 64, 16, True), (3, 257, 2, 1, 80, 5, False),
                                      (1, 300, 1, 2, 160, 8, True), (2, 200, 1, 1, 16, 4, True)):
        print("attention_kv8 tall", R, S, H, G, dh, W, causal, flush=True)
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
        print("attention_kv8 plan", R, S, Hq, H, dh, W, flush=True)
        pages, table = a_cache(S + W, R, W, H, dh)
        lens = [W * 64 - (W * 23 * r) % (W * 64) for r in range(R)]
        spoil(pages, table, lens)
        if i:
            table[0, W // 2] = -1
        q = rand(S + W, R, S, Hq * dh, dtype=(BF16, F16)[i])
        check_attention(q, pages, table, lens, dh ** -0.5, H, [n - S for n in lens] if i else None)


def test_attention_holes_and_bad_pages():
    R, H, dh, W = 3, 2, 64, 6
    pages, table = a_cache(1, R, W, H, dh)
    table[0, 1], table[0, 5], table[1, 0], table[2] = -1, 10 ** 6, -7, -1
    q = rand(1, R, 2, 4 * dh, dtype=F16)
    out = check_attention(q, pages, table, [384, 300, 384], dh ** -0.5, H)
    assert (out[2] == 0).all()
    assert (check_attention(q, pages, table, [-5, 0, 384], 0.1, H) == 0).all()
    check_attention(q, pages, table, [10 ** 9, 2 ** 31 - 1, 7], 0.1, H)  # cut to the table


def test_attention_value_scales_far_apart():
    """Pages whose values differ by more than a float16 operand holds, in either order."""
    for dtype in (F16, BF16):
        for order in ((100, 127, 145, 110, 127), (145, 100, 127, 1, 140), (1, 30, 60, 90, 120)):
            pages, table = a_cache(2, 1, 5, 1, 64)
            pages[3][table[0]] = np.array(order, np.uint8)[:, None]
            pages[2][:] = 118
            q = rand(3, 1, 3, 64, dtype=dtype)
            # results within the type: the largest scale's values times 448 stay below its limit
            if dtype == F16:
                pages[1][table[0]] &= 0x87  # small codes
            check_attention(q, pages, table, [320], 0.125, 1)


@pytest.mark.parametrize("S", [40, 150])
def test_attention_value_scales_far_apart_many_queries(S):
    """The same where queries share pages (64 and 128 of them): exponents up to 80 apart, no limit
    and a causal one."""
    for order in ((100, 127, 145, 110, 127), (145, 100, 127, 70, 140), (40, 60, 90, 119, 120)):
        pages, table = a_cache(2, 1, 5, 1, 64)
        pages[3][table[0]] = np.array(order, np.uint8)[:, None]
        pages[2][:] = 118
        q = rand(3, 1, S, 64, dtype=BF16)
        check_attention(q, pages, table, [320], 0.125, 1)
        check_attention(q, pages, table, [310], 0.125, 1, [310 - S])
    pages, table = a_cache(2, 320, 2, 1, 64)  # 320 rows: tiles of 128 queries for the larger S
    pages[3][table] = np.array([[145], [90]], np.uint8)
    pages[2][:] = 118
    check_attention(rand(3, 320, S - 50 if S > 64 else S, 64, dtype=BF16), pages, table, [120] * 320,
                    0.125, 1)


def test_attention_peaked_and_large_scores():
    """References that move late, scores of hundreds, one key that takes all."""
    for dtype in (F16, BF16):
        pages, table = a_cache(4, 2, 8, 1, 128)
        pages[2][table[0, 5]] += 6
        pages[2][table[1, 7]] += 9
        q = rand(5, 2, 20, 2 * 128, dtype=dtype)
        check_attention(q, pages, table, [512, 512], 0.1, 1)
        check_attention(q, pages, table, [512, 449], -0.1, 1)
        check_attention(q, pages, table, [512, 449], 0.0, 1)


@pytest.mark.parametrize("S", [9, 40, 200])
def test_attention_nan_reaches_only_who_sees_it(S):
    """A NaN key or value before some query's limit and behind another's; NaN scales."""
    for dtype in (F16, BF16):
        pages, table = a_cache(6, 1, 4, 1, 64)
        q = rand(7, 1, S, 64, dtype=dtype)
        first = 250 - S
        at = 250 - S // 2
        pages[1][table[0, at // 64], 0, 13, at % 64] = 0x7F
        pages[1][table[0, at // 64], 0, 37, at % 64] = 0xFF
        out = check_attention(q, pages, table, [251], 0.125, 1, [first])
        assert torch.isnan(out).any() and not torch.isnan(out[0, :S // 2]).any()
        pages[0][table[0, at // 64], 0, at % 64, 3] = 0x7F
        check_attention(q, pages, table, [251], 0.125, 1, [first])
        pages, table = a_cache(6, 1, 4, 1, 64)
        pages[3][table[0, 3]] = 255
        check_attention(q, pages, table, [251], 0.125, 1, [first])
        check_attention(q, pages, table, [192], 0.125, 1)
        pages[3][table[0, 3]], pages[2][table[0, 3]] = 120, 255
        check_attention(q, pages, table, [251], 0.125, 1, [first])


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


def test_attention_empty():
    pages = nv().nv_kv8_pages(3, 2, 64, "cuda")
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    q = rand(0, 2, 3, 128, dtype=F16)
    assert (nv().nv_op_attention_kv8(q, pages, z(2, 0), z(2), 0.1) == 0).all()
    assert nv().nv_op_attention_kv8(q[:, :0], pages, z(2, 1), z(2), 0.1).shape == (2, 0, 128)
    assert nv().nv_op_attention_kv8(q[:0], pages, z(0, 1), z(0), 0.1).shape == (0, 3, 128)
    nv().nv_op_kv8_append(q[:, :0], q[:, :0], pages, z(2, 1), z(2))
    nv().nv_op_kv8_append(q[:0], q[:0], pages, z(0, 1), z(0))


# ---------------------------------------------------------------------------------- together

class Layer:
    """norm -> q|k|v -> append -> attention -> output product + residual -> norm, on a cache."""

    def __init__(self, R, T, D, Hq, H, dh, W, dtype):
        self.Hq, self.H, self.dh, self.dtype = Hq, H, dh, dtype
        P = nv()
        self.w1, self.w2 = 1 + 0.1 * rand(1, D), 1 + 0.1 * rand(2, D)
        self.wqkv = P.nv_op_quant8(rand(3, (Hq + 2 * H) * dh, D, scale=D ** -0.5), block_rows=128)
        self.wo = P.nv_op_quant8(rand(4, D, Hq * dh, scale=(Hq * dh) ** -0.5), block_rows=128)
        self.pages = P.nv_kv8_pages(R * W, H, dh, "cuda")
        self.table = torch.randperm(R * W, generator=torch.Generator().manual_seed(5)).view(
            R, W).int().cuda()

    def __call__(self, x, r, pos, count):
        """x, r [R * T][D]; returns (codes, scales, h) of the next norm."""
        P, R = nv(), self.table.shape[0]
        C, Ck = self.Hq * self.dh, self.H * self.dh
        q, s, h = P.nv_op_rmsnorm8(x, self.w1, residual=r)
        qkv = P.nv_op_linear8(q, s, *self.wqkv, dtype=self.dtype).view(R, -1, C + 2 * Ck)
        P.nv_op_kv8_append(qkv[:, :, C:C + Ck], qkv[:, :, C + Ck:], self.pages, self.table, pos, count)
        a = P.nv_op_attention_kv8(qkv[:, :, :C], self.pages, self.table, pos + count,
                                  self.dh ** -0.5, qpos=pos)
        aq, as_ = P.nv_op_quant8(a.reshape(-1, C))
        y = P.nv_op_linear8(aq, as_, *self.wo, residual=h, dtype=self.dtype)
        return (qkv, a) + P.nv_op_rmsnorm8(y, self.w2, residual=h)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_layer_of_all_of_them(dtype):
    """A prompt, then single tokens, each step held to the oracle on that step's own inputs."""
    R, T, D, Hq, H, dh, W = 3, 100, 640, 10, 2, 64, 4
    layer = Layer(R, T, D, Hq, H, dh, W, dtype)
    pos = torch.zeros(R, dtype=torch.int32, device="cuda")
    for step, count in enumerate(([100, 37, 64], [1, 1, 1], [1, 0, 1], [1, 1, 1])):
        n = T if step == 0 else 1
        count = torch.tensor(count, dtype=torch.int32, device="cuda")
        x, r = rand(10 + step, R * n, D, dtype=dtype), rand(20 + step, R * n, D, dtype=dtype)
        was = [t.clone() for t in layer.pages]
        qkv, a, q2, s2, h2 = layer(x, r, pos, count)
        C, Ck = Hq * dh, H * dh
        tb, ps, cn = layer.table.cpu().numpy(), pos.cpu().numpy(), count.cpu().numpy()
        sh = lambda t: np64(t).reshape(R, n, H, dh)
        ok, oks = O.append(sh(qkv[:, :, C:C + Ck]), bits(was[0]), bits(was[2]), tb, ps, cn, False)
        ov, ovs = O.append(sh(qkv[:, :, C + Ck:]), bits(was[1]), bits(was[3]), tb, ps, cn, True)
        for g, w in zip(layer.pages, (ok, ov, oks, ovs)):
            assert np.array_equal(bits(g), w)
        o, spread, size, most = O.attention(np64(qkv[:, :, :C]).reshape(R, n, Hq, dh), ok, ov, oks, ovs,
                                            tb, ps + cn, dh ** -0.5, H, ps)
        rel = 2 * (dh * E * size + 8 * E * most + 4 * E) + 2 * u(F16) + u(dtype) + W * 64 * E
        assert (np.abs(np64(a).reshape(o.shape) - o) <= rel * spread + 1e-5).all()
        assert not torch.isnan(h2).any() and not ((bits(q2) & 127) == 127).any()
        # the whole step against float64 products of the same 8-bit operands: the first norm's
        # codes differ from the oracle's only where a value lies next to a code's edge
        y1 = O.rmsnorm(np64(x), np64(layer.w1), np64(r))
        full = O.values(*O.quantise(y1)) @ O.values(bits(layer.wqkv[0]), bits(layer.wqkv[1]), 128).T
        err = np.linalg.norm(np64(qkv).reshape(full.shape) - full) / np.linalg.norm(full)
        assert err <= 2 * u(dtype)
        pos = pos + count


def test_layer_on_another_stream_and_in_a_graph():
    """Single-token steps captured once and replayed: every replay equals the eager step."""
    R, D, Hq, H, dh, W = 4, 640, 8, 2, 128, 40
    eager, graph = (Layer(R, 1, D, Hq, H, dh, W, F16) for _ in range(2))
    for a, b in zip(eager.pages + (eager.table,) + eager.wqkv + eager.wo,
                    graph.pages + (graph.table,) + graph.wqkv + graph.wo):
        b.copy_(a)
    fill = torch.tensor([2400, 5, 64, 700], dtype=torch.int32, device="cuda")
    for layer in (eager, graph):  # a prompt's keys and values
        k, v = rand(1, R, 2400, H * dh, dtype=F16), rand(2, R, 2400, H * dh, dtype=F16)
        nv().nv_op_kv8_append(k, v, layer.pages, layer.table, fill * 0, fill)
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
    dev, tb = to_pages(pages), bytes_of(table)
    lens = torch.tensor([6400, 3001], dtype=torch.int32, device="cuda")
    q = rand(1, 2, 1, 8 * 128, dtype=F16)
    x, xs = P.nv_op_quant8(rand(2, 40, 4096))
    w, ws = P.nv_op_quant8(rand(3, 320, 4096), block_rows=128)
    a0, y0 = P.nv_op_attention_kv8(q, dev, tb, lens, 0.1), P.nv_op_linear8(x, xs, w, ws)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(5):
        with torch.cuda.stream(s1):
            got.append((P.nv_op_attention_kv8(q, dev, tb, lens, 0.1), P.nv_op_linear8(x, xs, w, ws)))
        with torch.cuda.stream(s2):
            got.append((P.nv_op_attention_kv8(q, dev, tb, lens, 0.1), P.nv_op_linear8(x, xs, w, ws)))
    torch.cuda.synchronize()
    for a, y in got:
        assert torch.equal(a, a0) and torch.equal(y, y0)
