"""The rotation of queries and keys and the 4-bit cache without a GPU: the oracle against values by
hand and against complex numbers, and every refusal of the C entry points and their Python wrappers
(nothing is launched)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import ops4 as O


def test_oracle_codes_round_to_the_nearest_even():
    ties = {0.25: 0, 0.75: 2, 1.25: 2, 1.75: 4, 2.5: 4, 3.5: 6, 5.0: 6}
    for x, c in ties.items():
        assert O.encode(x) == c and O.encode(-x) == c + 8
        assert O.encode(np.nextafter(x, 9)) == c + (c == np.searchsorted(O.POSITIVE, x) - 1)
        assert O.encode(np.nextafter(x, 0)) == c - (c == np.searchsorted(O.POSITIVE, x))
    assert np.array_equal(O.encode(O.VALUES), np.arange(16))  # code 8 is -0
    assert O.encode(-0.0) == 8
    rng = np.random.default_rng(0)
    x = rng.uniform(-6, 6, 5000)
    d = np.abs(x[:, None] - O.VALUES).min(1)
    assert np.array_equal(np.abs(x - O.VALUES[O.encode(x)]), d)


def test_oracle_scale_is_the_smallest_that_fits():
    rng = np.random.default_rng(1)
    a = np.concatenate([np.exp2(rng.uniform(-110, 120, 2000)), 6 * np.exp2(np.arange(-90., 90.)),
                        6 * np.exp2(np.arange(-90., 90.)) * (1 + 2 ** -23)])
    e = O.scale_byte(a)
    assert (a <= 6 * O.scale_value(e)).all()
    assert (a > 6 * O.scale_value(e - 1))[e > 1].all()
    assert O.scale_byte(0.0) == 1 and O.scale_byte(np.inf) == 255 and np.isnan(O.scale_value(255))


def test_oracle_bytes_and_blocks():
    x = np.zeros((2, 40))
    x[0, 0], x[0, 1], x[0, 39], x[1, 5], x[1, 33] = 6, -3, 1, np.nan, 12
    c, e = O.quantise(x)
    assert c.shape == (2, 20) and e.shape == (2, 2)
    assert c[0, 0] == 7 | 13 << 4 and list(e[0]) == [127, 125] and c[0, 19] == 6 << 4
    assert list(e[1]) == [255, 128] and not c[1, :16].any() and c[1, 16] == 7 << 4
    v = O.values(c, e)
    assert np.array_equal(v[0], x[0]) and np.isnan(v[1, :32]).all() and v[1, 33] == 12


def test_oracle_append_touches_its_own_tokens_only():
    rng = np.random.default_rng(2)
    codes = rng.integers(0, 256, (4, 2, 64, 8)).astype(np.uint8)
    scales = rng.integers(100, 130, (4, 2, 64, 1)).astype(np.uint8)
    x = rng.standard_normal((2, 3, 2, 16))
    table = np.array([[2, -1], [0, 3]])
    c, s = O.append(x, codes, scales, table, [62, -1], [3, 3])
    wc, ws = O.quantise(x[0, :2].transpose(1, 0, 2))
    assert np.array_equal(c[2, :, 62:], wc) and np.array_equal(s[2, :, 62:], ws)
    c[2, :, 62:], s[2, :, 62:] = codes[2, :, 62:], scales[2, :, 62:]
    assert np.array_equal(c, codes) and np.array_equal(s, scales)
    y = O.read(codes, scales, table, [63, 10], 2, [2, 1]).reshape(2, 2, 2, 16)
    assert np.array_equal(y[0, 0], O.values(codes[2, :, 63], scales[2, :, 63]))
    assert not y[0, 1].any() and not y[1, 1].any()


@pytest.mark.parametrize("halves", [False, True])
def test_oracle_rotation_is_a_product_of_complex_numbers(halves):
    rng = np.random.default_rng(3)
    x, axes = rng.standard_normal((2, 3, 2, 24)), (4, 10, 6)
    pos = rng.integers(-9, 9, (2, 3, 3))
    freqs = rng.uniform(0, 2, 10)
    y, _ = O.rope(x, pos, axes, freqs, halves=halves)
    at = p = 0
    for a, n in enumerate(axes):
        z, w = x[..., at:at + n], y[..., at:at + n]
        z, w = [(t[..., :n // 2] + 1j * t[..., n // 2:]) if halves else (t[..., ::2] + 1j * t[..., 1::2])
                for t in (z, w)]
        turn = np.exp(1j * pos[..., a, None] * freqs[p:p + n // 2])[:, :, None]
        assert np.allclose(w, z * turn, rtol=0, atol=1e-14)
        at, p = at + n, p + n // 2
    assert np.array_equal(y[..., 20:], x[..., 20:])


# ------------------------------------------------------------------------------- refusals

D = C.c_void_p(0x10000)      # never read: every call here ends before a launch
ODD = C.c_void_p(0x10004)


def _lib():
    from paper_2312_04429_amd import _native as N
    return N


def test_rope_refusals():
    N = _lib()

    def call(q=D, ldq=256, qr=256, qo=D, ldqo=256, qor=256, qh=4, qw=None, k=D, ldk=128, kr=128, ko=D,
             ldko=128, kor=128, kh=2, kw=None, dt=N.NV_F16, rows=2, S=3, dh=64, pos=D, ldp=2, pr=6,
             axes=(16, 48), freqs=D, halves=0, norm=1, eps=1e-6, n=None):
        ax = None if axes is None else (C.c_int32 * max(1, len(axes)))(*axes)
        return N.lib.nv_op_qk_rope(q, ldq, qr, qo, ldqo, qor, qh, qw, k, ldk, kr, ko, ldko, kor, kh, kw,
                                   dt, rows, S, dh, pos, ldp, pr,
                                   (0 if axes is None else len(axes)) if n is None else n, ax, freqs,
                                   halves, norm, eps, None)
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(pos=None),
                dict(freqs=None), dict(dt=N.NV_F32), dict(dt=9), dict(rows=-1), dict(S=-1), dict(qh=-1),
                dict(kh=-1), dict(axes=(15, 48)), dict(axes=(-2, 8)), dict(axes=(32, 34)),
                dict(axes=(2147483646, 2147483646, 4)), dict(axes=None, n=2), dict(n=-1), dict(halves=2),
                dict(norm=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(norm=0, qw=D), dict(norm=0, kw=D), dict(ldqo=255), dict(ldko=127), dict(ldq=-1),
                dict(ldk=-1), dict(qr=-1), dict(kr=-1), dict(qor=-1), dict(kor=-1), dict(ldp=-1),
                dict(pr=-1)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    for bad in (dict(dh=60), dict(dh=0), dict(dh=-8), dict(dh=264), dict(axes=(2, 2, 2, 2, 2)),
                dict(rows=1 << 30, S=1 << 30), dict(qh=1 << 20, ldqo=1 << 26)):
        assert call(**bad) == N.NV_ERR_UNSUPPORTED, bad
    for ok in (dict(rows=0), dict(S=0), dict(qh=0, kh=0), dict(S=0, axes=(), pos=None, freqs=None)):
        assert call(**ok) == N.NV_OK, ok


def test_append_refusals():
    N = _lib()

    def call(k=D, v=D, ld=64, rs=64, dt=N.NV_F16, rows=1, T=1, H=1, dh=64, kp=D, vp=D, ks=D, vs=D,
             n=4, table=D, W=4, pos=D, count=None):
        return N.lib.nv_op_kv4_append(k, ld, rs, v, ld, rs, dt, rows, T, H, dh, kp, vp, ks, vs, n,
                                      table, W, pos, count, None)
    for bad in (dict(k=None), dict(v=None), dict(kp=None), dict(vp=None), dict(ks=None),
                dict(vs=None), dict(table=None), dict(pos=None), dict(dt=N.NV_F32), dict(rows=-1),
                dict(rows=65536), dict(T=-1), dict(H=0), dict(H=32768), dict(n=-1), dict(W=-1),
                dict(ld=-1), dict(rs=-1), dict(kp=ODD), dict(vp=ODD)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    for bad in (dict(dh=48), dict(dh=0), dict(dh=-64), dict(dh=256), dict(T=1 << 29)):
        assert call(**bad) == N.NV_ERR_UNSUPPORTED, bad
    for ok in (dict(rows=0), dict(T=0), dict(n=0), dict(W=0)):
        assert call(**ok) == N.NV_OK, ok


def test_read_refusals():
    N = _lib()

    def call(kp=D, vp=D, ks=D, vs=D, n=4, table=D, W=4, pos=D, count=None, rows=1, T=1, H=2, dh=64, k=D,
             v=D, ld=128, rs=128, dt=N.NV_F32):
        return N.lib.nv_op_kv4_read(kp, vp, ks, vs, n, table, W, pos, count, rows, T, H, dh, k, ld, rs,
                                    v, ld, rs, dt, None)
    for bad in (dict(k=None), dict(v=None), dict(kp=None), dict(vp=None), dict(ks=None),
                dict(vs=None), dict(table=None), dict(pos=None), dict(dt=5), dict(rows=-1),
                dict(rows=65536), dict(T=-1), dict(H=0), dict(H=32768), dict(n=-1), dict(W=-1),
                dict(ld=127), dict(rs=-1), dict(kp=ODD), dict(vp=ODD)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    for bad in (dict(dh=48), dict(dh=-8), dict(T=1 << 30)):
        assert call(**bad) == N.NV_ERR_UNSUPPORTED, bad
    assert call(rows=0) == N.NV_OK and call(T=0) == N.NV_OK


def test_attention_kv4_refusals():
    N = _lib()

    def call(q=D, ldq=256, qr=256, dt=N.NV_F16, kp=D, vp=D, ks=D, vs=D, n=4, table=D, W=4, lens=D,
             qpos=None, rows=1, S=1, H=4, G=2, dh=64, scale=1.0, out=D, ldo=256, orow=256, wsp=None,
             wsb=0):
        return N.lib.nv_op_attention_kv4(q, ldq, qr, dt, kp, vp, ks, vs, n, table, W, lens, qpos, rows,
                                         S, H, G, dh, scale, out, ldo, orow, wsp, wsb, None)
    for bad in (dict(q=None), dict(kp=None), dict(vp=None), dict(ks=None), dict(vs=None),
                dict(table=None), dict(lens=None), dict(out=None), dict(dt=N.NV_F32), dict(rows=-1),
                dict(S=-1), dict(H=0), dict(G=0), dict(H=3), dict(n=-1), dict(W=-1), dict(W=1 << 25),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(ldo=255), dict(ldq=-8),
                dict(qr=-8), dict(orow=-8), dict(kp=ODD), dict(vp=ODD)):
        assert call(**bad) == N.NV_ERR_INVALID_ARG, bad
    for bad in (dict(dh=48), dict(ldq=252), dict(qr=4), dict(ldo=260), dict(orow=4), dict(q=ODD),
                dict(out=ODD)):
        assert call(**bad) == N.NV_ERR_UNSUPPORTED, bad
    assert call(rows=0) == N.NV_OK and call(S=0) == N.NV_OK
    need = N.lib.nv_op_attention_kv4_workspace(1, 1, 4, 2, 64, 1000)
    assert need > 0
    assert call(W=1000, wsb=need - 1) == N.NV_ERR_WORKSPACE
    assert call(W=1000, wsp=D, wsb=need - 1) == N.NV_ERR_WORKSPACE
    assert call(W=1000, wsp=None, wsb=need) == N.NV_ERR_WORKSPACE
    assert call(W=1000, wsp=ODD, wsb=need) == N.NV_ERR_WORKSPACE
    assert N.lib.nv_op_attention_kv4_workspace(1, 1, 4, 3, 64, 1000) == 0


def test_attention_kv4_more_queries_than_64_bits_count():
    N = _lib()
    for rows, S, H, G in ((1, 1 << 30, 1 << 10, 1), (1 << 30, 1 << 30, 1 << 30, 1 << 30),
                          (1, (1 << 31) - 1, 1, 1), (1 << 30, 1 << 20, 64, 1)):
        st = N.lib.nv_op_attention_kv4(D, H * 16, 0, N.NV_F16, D, D, D, D, 4, D, 64, D, None, rows, S,
                                       H, G, 16, 1.0, D, H * 16, 0, D, 1 << 20, None)
        assert st == N.NV_ERR_UNSUPPORTED, (rows, S, H, G)


def test_wrappers_take_device_tensors_only():
    import paper_2312_04429_amd as P
    x = torch.zeros(1, 2, 64, dtype=torch.float16)
    pages = P.nv_kv4_pages(2, 1, 40, "cpu")
    assert [tuple(t.shape) for t in pages] == [(2, 1, 64, 20)] * 2 + [(2, 1, 64, 2)] * 2
    f = P.nv_rope_freqs((4, 6), 100.0, "cpu")
    assert f.dtype == torch.float64 and torch.allclose(
        f, torch.tensor([1, 0.1, 1, 100 ** (-1 / 3), 100 ** (-2 / 3)], dtype=torch.float64))
    i = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: P.nv_op_qk_rope(x, x, 64, i[None, None], (64,), f),
                 lambda: P.nv_op_kv4_append(x, x, pages, i[None], i),
                 lambda: P.nv_op_kv4_read(pages, i[None], i, 1),
                 lambda: P.nv_op_attention_kv4(x, pages, i[None], i, 1.0)):
        with pytest.raises(ValueError, match="device"):
            call()
