"""Attention over the 8-bit cache where values, scores or sums are far from one another in size, against
float64; the bound of each output is derived beside the helper that computes it."""
import numpy as np
import pytest
import torch

import ops8_values as V
from oracle import ops8 as O

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# rows, queries: tiles of 16 with shares and without, of 64 and of 128
PLANS = [(1, 3), (300, 3), (1, 40), (600, 40), (1, 150), (600, 150)]


def nv():
    import paper_2312_04429_amd as P
    return P


def run(q, pages, table, lens, scale, qpos=None, rows=1, dtype="bf16"):
    """The call on `rows` rows that read the same pages: [S][Hq][dh] of the first; the others are equal
    to the bit."""
    _, S, Hq, dh = q.shape
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    rep = lambda a: dev(np.repeat(np.asarray(a, np.int32), rows, 0))
    x = dev(q).to(TYPES[dtype]).reshape(1, S, Hq * dh).expand(rows, S, Hq * dh)
    out = nv().nv_op_attention_kv8(x, tuple(dev(p) for p in pages), rep(table), rep(lens), scale,
                                   qpos=None if qpos is None else rep(qpos))
    assert (out.view(torch.int16) == out[:1].view(torch.int16)).all()
    return out[0].double().cpu().numpy().reshape(S, Hq, dh)


def check(q, pages, table, lens, scale, qpos=None, rows=1, dtype="bf16"):
    print("attention_kv8", rows, q.shape, table.shape, lens, qpos, dtype, flush=True)
    o, tol = V.attention(q, pages, table, lens, scale, qpos, dtype)
    got = run(q, pages, table, lens, scale, qpos, rows, dtype)
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got - o[0]) <= tol[0])
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(),
                               float(np.nanmax(np.abs(got - o[0]) / tol[0])))
    return o[0], got


# ------------------------------------------------------------------------- values near the type's end

@pytest.mark.parametrize("W", [5, 40, 320])
@pytest.mark.parametrize("rows,S", PLANS)
def test_sums_of_large_values(rows, S, W):
    """Values of 2^120: their sum over the row passes float32, their mean does not."""
    dh, rng = 64, np.random.default_rng(W)
    kp = V.codes(rng, (W, 1, 64, dh), 0x20, 0x40)
    vp = rng.integers(0x30, 0x39, (W, 1, dh, 64)).astype(np.uint8)
    pages = [kp, vp, np.full((W, 1), 122, np.uint8), np.full((W, 1), 247, np.uint8)]
    table = rng.permutation(W).reshape(1, W).astype(np.int32)
    o, _ = check(V.queries(S, 1, dh), pages, table, [W * 64 - 7], 0.125, rows=rows)
    assert o.min() > 2.0 ** 119


# ---------------------------------------------------------------------- scales that a query does not see

@pytest.mark.parametrize("order", ["last", "middle"])
@pytest.mark.parametrize("rows,S", [(1, 5), (300, 5), (1, 60), (600, 60), (1, 120), (600, 120)])
def test_scales_behind_the_limit_leave_a_query_alone(rows, S, order):
    """Some queries of a tile see a page whose values are 2^150 times those before it, the others end
    before it: theirs are the bits of a call without that page."""
    pages, table = V.far_cache(150, order, top=250)
    first = 64 * V.ORDERS[order].index(0)            # token where the large page begins
    q, n = V.queries(S, 1, 64), 64 * table.shape[1]
    qpos = [first - S // 2]                          # queries 0 .. S // 2 - 1 end before it
    _, got = check(q, pages, table, [n], 0.125, qpos, rows)
    o, alone = check(q, pages, table, [first], 0.125, qpos, rows)
    assert np.array_equal(got[:S // 2], alone[:S // 2]) and (o[:S // 2] != 0).all()


@pytest.mark.parametrize("rows,S", [(1, 60), (600, 60), (1, 120), (600, 120)])
def test_nan_page_beside_scales_behind_the_limit(rows, S):
    """The same with a NaN value in the last page that all queries see part of: it waits for the end."""
    pages, table = V.far_cache(150, "last", top=250)
    q = V.queries(S, 1, 64)
    pages[1][table[0, 3], 0, 50, 63] = 0x7F          # token 255: seen by the second half
    qpos = [256 - S // 2 - 1]
    o, tol = V.attention(q, pages, table, [320], 0.125, qpos)
    got = run(q, pages, table, [320], 0.125, qpos, rows)
    assert np.array_equal(np.isnan(got), np.isnan(o[0])) and np.isnan(got).any()
    with np.errstate(invalid="ignore"):
        assert not (np.abs(got - o[0]) > tol[0]).any()
    assert (got[:S // 2, 0, :50] != 0).all()


# --------------------------------------------------------------------------- value scales far apart

@pytest.mark.parametrize("order", sorted(V.ORDERS))
@pytest.mark.parametrize("rows,S", PLANS)
def test_value_scales_far_apart(rows, S, order):
    """Channels that only pages far below the largest scale decide, that page before and behind."""
    for d in V.DISTANCES:
        pages, table = V.far_cache(d, order)
        q = V.queries(S, 1, 64)
        n = 64 * table.shape[1]
        check(q, pages, table, [n], 0.125, rows=rows)
        check(q, pages, table, [n - 2], 0.125, [n - 2 - S], rows=rows)


# ------------------------------------------------------------------------------- small probabilities

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,S", PLANS)
def test_tail_below_one_key(rows, S, dtype):
    """One key far above all others, its value zero: the others' small probabilities are the result.
    Flat tails, a tail that spreads, the key in the first page and behind."""
    for at in (0, 3 * 64 + 9):
        for bits, spread in V.TAILS:
            q, pages, table, n, scale = V.tail_cache(S, at, bits, spread)
            check(q, pages, table, [n], scale, rows=rows, dtype=dtype)


# ------------------------------------------------------------------------------------- large scores

@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("rows,S", PLANS)
def test_scores_of_any_size_pick_the_largest(rows, S, sign):
    """Scores up to 2^40 whose neighbours lie far apart: the result is the value of one key, of either sign
    of the scores, wherever that key is, and however the sum of a score and a small number rounds."""
    dh, W = 64, 9
    rng = np.random.default_rng(7)
    table = rng.permutation(W).reshape(1, W).astype(np.int32)
    vp = V.codes(rng, (W, 1, dh, 64), 0x20, 0x50)
    q = np.zeros((1, S, 1, dh))
    q[..., 0] = 1
    for at in (5, 300, W * 64 - 1):
        kp = np.zeros((W, 1, 64, dh), np.uint8)
        kp[..., 0] = rng.integers(0x70, 0x7A, (W, 1, 64))          # 128 .. 320
        kp[table[0, at // 64], 0, at % 64, 0] = 0x7E if sign > 0 else 0x68   # 448, 64
        pages = [kp, vp, np.full((W, 1), 127, np.uint8), np.full((W, 1), 127, np.uint8)]
        want = O.VALUES[vp[table[0, at // 64], 0, :, at % 64]]
        for e in range(10, 41):
            for m in (1.0, 1.13, 1.37, 1.71):
                got = run(q, pages, table, [W * 64], sign * m * 2.0 ** e / 448, rows=rows, dtype="f16")
                assert (got == want).all(), (at, e, m)


@pytest.mark.parametrize("d", [20, 64, 65, 100, 120])
@pytest.mark.parametrize("rows,S", [(1, 5), (300, 5), (1, 60), (600, 60), (1, 120), (600, 120)])
def test_nan_page_beside_pages_far_below(rows, S, d):
    """Both kinds of pages that may wait for the end of the loop, in one row and in one page, with a hole
    between them."""
    for at in (2, 4):
        pages, table = V.far_cache(d, "first")
        table[0, 3 if at == 4 else 1] = -1
        pages[1][table[0, at], 0, 50, 63] = 0xFF
        end = 64 * at + 64                           # the NaN's token is end - 1: the later half sees it
        q, qpos = V.queries(S, 1, 64), [end - S // 2 - 1]
        o, tol = V.attention(q, pages, table, [end], 0.125, qpos)
        got = run(q, pages, table, [end], 0.125, qpos, rows)
        assert np.array_equal(np.isnan(got), np.isnan(o[0])) and np.isnan(got).any()
        with np.errstate(invalid="ignore"):
            assert not (np.abs(got - o[0]) > tol[0]).any()
