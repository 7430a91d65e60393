"""The 8-bit operators without a GPU: the oracle's 8-bit form against torch's own e4m3 type, and
every refusal of the C entry points and their Python wrappers (nothing is launched)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import ops8 as O
from ops8_sizes import FORM_SIZES, PLAN_SIZES


def test_oracle_codes_are_torchs_e4m3():
    codes = torch.arange(256, dtype=torch.uint8)
    v = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, O.VALUES, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 0.02,
                        O.VALUES[:127], (O.VALUES[:126] + O.VALUES[1:127]) / 2, [-0.0, np.nan]])
    x = x.astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = O.encode(x)
    assert np.array_equal(got & 127, t & 127)
    assert np.array_equal(got[~np.isnan(x)], t[~np.isnan(x)])


def test_oracle_scale_is_the_smallest_that_fits():
    rng = np.random.default_rng(1)
    a = np.concatenate([np.exp2(rng.uniform(-110, 120, 2000)), 448 * np.exp2(np.arange(-90., 90.)),
                        448 * np.exp2(np.arange(-90., 90.)) * (1 + 2 ** -23)])
    e = O.scale_byte(a)
    assert (a <= 448 * O.scale_value(e)).all()
    assert (a > 448 * O.scale_value(e - 1))[e > 1].all()
    assert O.scale_byte(0.0) == 1 and np.isnan(O.scale_value(255))


def test_oracle_append_keeps_what_it_should():
    rng = np.random.default_rng(2)
    codes, scales = rng.integers(0, 120, (4, 1, 64, 16)).astype(np.uint8), np.full((4, 1), 120, np.uint8)
    x = rng.standard_normal((1, 3, 1, 16))
    c, s = O.append(x, codes, scales, np.array([[2, -1]]), [62], [3], False)
    assert np.array_equal(c[[0, 1, 3]], codes[[0, 1, 3]]) and np.array_equal(s[[0, 1, 3]], scales[[0, 1, 3]])
    assert np.array_equal(c[2, 0, 62:], O.encode(x[0, :2, 0] * 2.0 ** (127 - int(s[2, 0]))))


# ------------------------------------------------------------------------------- refusals

D = C.c_void_p(0x10000)      # never read: every call here ends before a launch
ODD = C.c_void_p(0x10004)


def _lib():
    from paper_2312_04429_amd import _native as N
    return N


def test_quant8_refusals():
    N = _lib()

    def call(x=D, dt=N.NV_F16, ldx=256, M=4, K=256, br=1, q=D, ldq=256, s=D):
        return N.lib.nv_op_quant8(x, dt, ldx, M, K, br, q, ldq, s, None)
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(dt=7), dict(M=-1), dict(K=0),
                dict(br=2), dict(ldx=255), dict(ldq=255)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    assert call(M=0, x=None) == N.NV_OK

    def back(q=D, ldq=256, s=D, M=4, K=256, br=1, out=D, dt=N.NV_F16, ldo=256):
        return N.lib.nv_op_dequant8(q, ldq, s, M, K, br, out, dt, ldo, None)
    for bad in (dict(q=None), dict(s=None), dict(out=None), dict(dt=-1), dict(M=-1), dict(K=0),
                dict(br=0), dict(ldq=1), dict(ldo=255)):
        assert back(**bad) == N.NV_ERR_INVALID_ARG, bad
    assert back(M=0) == N.NV_OK


def test_quant8_rows_past_32_bit_columns():
    N = _lib()
    K = (1 << 31) - 1
    for br in (1, 128):
        assert N.lib.nv_op_quant8(D, N.NV_F16, K, 1, K, br, D, K, D, None) == N.NV_ERR_UNSUPPORTED
        assert N.lib.nv_op_dequant8(D, K, D, 1, K, br, D, N.NV_F16, K, None) == N.NV_ERR_UNSUPPORTED
    ok = (1 << 31) - 256
    assert N.lib.nv_op_quant8(D, N.NV_F16, ok, 0, ok, 1, D, ok, D, None) == N.NV_OK


def test_rmsnorm8_refusals():
    N = _lib()

    def call(x=D, ldx=64, r=None, ldr=0, dt=N.NV_F16, w=D, eps=1e-6, M=2, Dm=64, h=None, ldh=0, q=D,
             ldq=64, s=D):
        return N.lib.nv_op_rmsnorm8(x, ldx, r, ldr, dt, w, eps, M, Dm, h, ldh, q, ldq, s, None)
    for bad in (dict(x=None), dict(w=None), dict(q=None), dict(s=None), dict(dt=N.NV_F32),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(M=-1),
                dict(Dm=0), dict(ldx=63), dict(ldq=63), dict(r=D, ldr=63), dict(h=D, ldh=63)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    assert call(Dm=32769, ldx=40000, ldq=40000) == N.NV_ERR_UNSUPPORTED
    assert call(M=0) == N.NV_OK


def test_linear8_refusals():
    N = _lib()

    def call(x=D, ldx=256, xs=D, w=D, ldw=256, ws=D, b=None, r=None, ldr=0, out=D, ldo=64,
             dt=N.NV_F16, M=4, Nn=64, K=256):
        return N.lib.nv_op_linear8(x, ldx, xs, w, ldw, ws, b, r, ldr, out, ldo, dt, M, Nn, K, None)
    for bad in (dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(out=None),
                dict(dt=N.NV_F32), dict(M=-1), dict(M=1 << 31), dict(Nn=0), dict(K=0),
                dict(ldx=240), dict(ldw=240), dict(ldo=63), dict(r=D, ldr=63)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    for bad in (dict(ldx=264), dict(ldw=264), dict(x=ODD), dict(w=ODD), dict(ldx=(1 << 22) + 16)):
        assert call(**bad) == N.NV_ERR_UNSUPPORTED, bad
    assert call(M=0) == N.NV_OK
    assert call(M=(1 << 31) - 1, Nn=1 << 30, ldo=1 << 30) == N.NV_ERR_UNSUPPORTED


def test_append_refusals():
    N = _lib()

    def call(k=D, v=D, ld=64, rs=64, dt=N.NV_F16, rows=1, T=1, H=1, dh=64, kp=D, vp=D, ks=D, vs=D,
             n=4, table=D, W=4, pos=D, count=None):
        return N.lib.nv_op_kv8_append(k, ld, rs, v, ld, rs, dt, rows, T, H, dh, kp, vp, ks, vs, n,
                                      table, W, pos, count, None)
    for bad in (dict(k=None), dict(v=None), dict(kp=None), dict(vp=None), dict(ks=None),
                dict(vs=None), dict(table=None), dict(pos=None), dict(dt=N.NV_F32), dict(rows=-1),
                dict(rows=65536), dict(T=-1), dict(H=0), dict(H=40000), dict(n=-1), dict(W=-1),
                dict(ld=-8), dict(rs=-8), dict(kp=ODD), dict(vp=ODD)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    assert call(dh=48) == N.NV_ERR_UNSUPPORTED
    for empty in (dict(rows=0), dict(T=0), dict(n=0), dict(W=0)):
        assert call(**empty) == N.NV_OK, empty


def test_attention_kv8_refusals():
    N = _lib()

    def call(q=D, ldq=256, qr=256, dt=N.NV_F16, kp=D, vp=D, ks=D, vs=D, n=4, table=D, W=4, lens=D,
             qpos=None, rows=1, S=1, H=4, Hk=2, dh=64, scale=0.1, out=D, ldo=256, orow=256, wsp=D,
             wsb=1 << 40):
        return N.lib.nv_op_attention_kv8(q, ldq, qr, dt, kp, vp, ks, vs, n, table, W, lens, qpos,
                                         rows, S, H, Hk, dh, scale, out, ldo, orow, wsp, wsb, None)
    for bad in (dict(q=None), dict(lens=None), dict(out=None), dict(table=None), dict(kp=None),
                dict(vp=None), dict(ks=None), dict(vs=None), dict(dt=N.NV_F32), dict(rows=-1),
                dict(S=-1), dict(H=0), dict(Hk=0), dict(Hk=3), dict(n=-1), dict(W=-1),
                dict(W=1 << 25), dict(scale=float("nan")), dict(scale=float("inf")), dict(ldq=-8),
                dict(qr=-8), dict(ldo=248), dict(orow=-8), dict(kp=ODD), dict(vp=ODD)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    for bad in (dict(dh=48), dict(ldq=260), dict(qr=260), dict(ldo=260), dict(orow=4), dict(q=ODD),
                dict(out=ODD), dict(rows=1 << 30, S=1 << 20)):
        assert call(**bad) == N.NV_ERR_UNSUPPORTED, bad
    assert call(rows=0) == N.NV_OK and call(S=0) == N.NV_OK
    need = N.lib.nv_op_attention_kv8_workspace(1, 1, 4, 2, 64, 1000)
    assert need > 0
    assert call(W=1000, wsb=need - 1) == N.NV_ERR_WORKSPACE
    assert call(W=1000, wsp=None) == N.NV_ERR_WORKSPACE
    assert call(W=1000, wsp=ODD) == N.NV_ERR_WORKSPACE
    assert N.lib.nv_op_attention_kv8_workspace(1, 1, 4, 3, 64, 1000) == 0


def test_attention_kv8_more_queries_than_64_bits_count():
    # tiles of queries that are a multiple of 2^32, and products past 2^63: refused, nothing raised
    N = _lib()
    for rows, S, H, G in ((1, 1 << 30, 1 << 10, 1), (1 << 30, 1 << 30, 1 << 30, 1 << 30),
                          (1, (1 << 31) - 1, 1, 1), (1 << 30, 1 << 20, 64, 1)):
        assert N.lib.nv_op_attention_kv8_workspace(rows, S, H, G, 16, 64) == 0
        st = N.lib.nv_op_attention_kv8(D, H * 16, 0, N.NV_F16, D, D, D, D, 4, D, 64, D, None, rows, S,
                                       H, G, 16, 1.0, D, H * 16, 0, D, 1 << 20, None)
        assert st == N.NV_ERR_UNSUPPORTED, (rows, S, H, G)


def test_wrappers_take_device_tensors_only():
    import paper_2312_04429_amd as P
    x, s = torch.zeros(2, 128, dtype=torch.float16), torch.zeros(2, 1, dtype=torch.uint8)
    q = torch.zeros(2, 128, dtype=torch.uint8)
    pages = P.nv_kv8_pages(2, 1, 64, "cpu")
    assert [tuple(t.shape) for t in pages] == [(2, 1, 64, 64), (2, 1, 64, 64), (2, 1), (2, 1)]
    i = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: P.nv_op_quant8(x), lambda: P.nv_op_dequant8(q, s),
                 lambda: P.nv_op_rmsnorm8(x, torch.ones(128)),
                 lambda: P.nv_op_linear8(q, s, q, s),
                 lambda: P.nv_op_kv8_append(x[None], x[None], pages, i[None], i),
                 lambda: P.nv_op_attention_kv8(x[None], pages, i[None], i, 1.0)):
        with pytest.raises(ValueError, match="device"):
            call()


# ---------------------------------------------------------------------- the rules, on their own

@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("ops8")
    src, out = str(d / "rule.cpp"), str(d / "rule.so")
    with open(src, "w") as f:
        f.write('''
#include "kv8.h"
#include "linear8.h"
extern "C" int form(long long M, int N, int K) { return nv::linear8_form(M, N, K); }
extern "C" int forms() { return nv::L8_COUNT; }
extern "C" int few() { return nv::KV8_FEW; }
extern "C" void plan(long long rows, int S, int heads, int kv_heads, int dh, int pages, int* out) {
  const nv::Kv8Plan p = nv::kv8_plan(rows, S, heads, kv_heads, dh, pages);
  out[0] = p.tall, out[1] = p.splits, out[2] = p.col_tiles;
}
''')
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                        "paper_2312_04429_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", csrc,
                    src, "-o", out], check=True)
    lib = C.CDLL(out)
    lib.form.argtypes = [C.c_longlong, C.c_int, C.c_int]
    return lib


def test_every_form_of_the_product_is_reached(rules):
    assert sorted(FORM_SIZES) == list(range(rules.forms()))
    for form, sizes in FORM_SIZES.items():
        for s in sizes:
            assert rules.form(*s) == form, s


def _plan(rules, rows, *sizes):
    out = (C.c_int * 3)()
    rules.plan(C.c_longlong(rows), *sizes, out)
    return tuple(out)


def test_every_tile_and_join_of_attention_is_reached(rules):
    kind = lambda n: "one" if n == 1 else "few" if n <= rules.few() else "many"
    for want, sizes in PLAN_SIZES.items():
        for s in sizes:
            tall, splits, tiles = _plan(rules, *s)
            assert (tall, kind(splits)) == want, s
            assert tiles == -(-s[1] * (s[2] // s[3]) // (16, 64, 128)[tall])


def test_shares_of_attention_stay_in_bounds(rules):
    """At most 256 shares (the join's threads), 1024 workgroups of shares, and a page a share."""
    rng = np.random.default_rng(0)
    for _ in range(4000):
        rows, kv, group = (int(2 ** rng.uniform(0, t)) for t in (9, 6, 5))
        S, W = int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 20))
        dh = int(rng.choice([16, 32, 40, 64, 80, 128, 160]))
        tall, splits, tiles = _plan(rules, rows, S, kv * group, kv, dh, W)
        assert 1 <= splits <= 256 and (splits == 1 or splits <= W)
        assert splits == 1 or splits * tiles * rows * kv <= 1024, (rows, S, kv, group, dh, W)
        assert (tall > 0) == (S * group > 32) and tiles * (16, 64, 128)[tall] >= S * group


# us of each form (0 .. 7 as in linear8.h; None: not taken or not timed), graph-timed on one MI355X
TIMINGS = [
    (8, 1280, 5120, [7.3, 7.4, 10.7, 11.3, 13.9, 19.9, 19.0, None]),
    (16, 320, 5120, [8.7, 7.4, 10.6, 11.4, 13.8, 19.6, 18.9, None]),
    (16, 10240, 1280, [8.5, 9.5, 5.8, 6.1, 6.9, 9.2, 8.7, None]),
    (32, 1280, 5120, [None, 7.5, 10.9, 11.5, 14.1, 20.1, 18.8, None]),
    (64, 640, 640, [None, 5.9, 4.9, 5.1, 6.0, 8.1, 6.9, None]),
    (128, 5120, 1280, [None, 13.6, 7.5, 6.4, 7.7, 10.6, 9.2, None]),
    (256, 1280, 5120, [None, 16.4, 12.1, 13.5, 18.5, 33.6, 21.2, None]),
    (256, 10240, 640, [None, 37.5, 11.6, 10.0, 8.6, 9.3, 8.2, None]),
    (512, 2560, 2560, [None, 27.4, 13.1, 12.8, 12.1, 20.5, 14.9, None]),
    (512, 5120, 640, [None, 37.9, 11.5, 10.1, 8.8, 9.3, 8.2, None]),
    (1024, 1280, 1280, [None, 21.8, 8.5, 8.3, 8.4, 10.7, 9.4, 24.2]),
    (1024, 5120, 1280, [None, 82.3, 26.8, 20.8, 18.0, 16.2, 19.6, 26.6]),
    (2000, 1280, 5120, [None, 69.5, 37.2, 30.4, 28.2, 34.5, 22.9, 57.5]),
    (2000, 2560, 1280, [None, 84.3, 26.8, 21.2, 17.9, 16.3, 19.3, 26.2]),
    (4096, 1280, 1280, [None, 84.8, 26.8, 20.6, 18.2, 16.5, 20.1, 26.3]),
    (4096, 5120, 640, [None, 294.9, 67.6, 50.6, 36.4, 31.3, 34.7, 39.4]),
    (4096, 10240, 1280, [None, 657.6, 164.2, 131.3, 94.3, 75.2, 94.0, 78.6]),
    (8192, 640, 2560, [None, 104.0, 39.0, 28.7, 25.2, 23.1, 28.3, 36.6]),
    (8192, 2560, 2560, [None, 405.7, 128.9, 101.4, 80.6, 67.4, 76.3, 73.6]),
    (8192, 10240, 5120, [None, 2229.4, 851.1, 704.2, 585.5, 428.5, 496.5, 363.1]),
]


@pytest.mark.parametrize("M,N,K,us", TIMINGS)
def test_choice_of_form_is_near_the_fastest(M, N, K, us, rules):
    pick = us[rules.form(M, N, K)]
    assert pick is not None and pick <= 1.19 * min(t for t in us if t)
