"""Attention over the 4-bit cache where scores or values are far from one another in size, against what the
definition gives."""
import numpy as np
import pytest
import torch

from oracle import ops4 as O

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
# rows, queries, pages a row: tiles of 16 in one share, of more workgroups than are resident, in many shares; of
# 64 in one and in a few shares; of 128
PLANS = [(1, 3, 9), (600, 3, 9), (1, 40, 9), (1, 3, 40), (1, 300, 9), (1, 300, 40), (300, 300, 9)]


def nv():
    import paper_2312_04429_amd as P
    return P


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def run(q, pages, table, lens, scale, qpos=None, rows=1):
    """The call on `rows` rows that read the same pages, q [S][heads * dh] on the device: [S][heads * dh] of
    the first row; the others are equal to the bit."""
    rep = lambda a: dev(np.repeat(np.asarray(a, np.int32), rows, 0))
    out = nv().nv_op_attention_kv4(q.expand(rows, *q.shape), tuple(dev(p) for p in pages), rep(table), rep(lens),
                                   scale, qpos=None if qpos is None else rep(qpos))
    assert (out.view(torch.int16) == out[:1].view(torch.int16)).all()
    return out[0]


# ------------------------------------------------------------------------------------- large scores

@pytest.mark.parametrize("way", ["window", "beyond"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("rows,S,W", PLANS)
def test_scores_of_any_size_pick_the_largest(rows, S, W, sign, way):
    """Scores up to 2^40, the next ones a sixth of 2^e (170 at 2^10) and more below the largest: the result
    is the value of one key, of either sign of the scores, wherever that key is, and however the product of a
    score and the scale rounds.  beyond: that key's page has a value that float16 operands do not hold."""
    dh = 64
    print("attention_kv4 scores", rows, S, W, sign, way, flush=True)
    rng = np.random.default_rng(7)
    table = rng.permutation(W).reshape(1, W).astype(np.int32)
    vp = rng.integers(0, 256, (W, 1, 64, dh // 2)).astype(np.uint8)
    q = torch.zeros(S, dh, dtype=F16, device="cuda")
    q[:, 0] = 1 + torch.arange(S, device="cuda") % 61 / 64  # scores of more bits than a product keeps
    for at in (5, 300, W * 64 - 1):
        page, slot = table[0, at // 64], at % 64
        kp = np.zeros((W, 1, 64, dh // 2), np.uint8)
        kp[..., 0] = rng.integers(4, 7, (W, 1, 64))        # 2, 3, 4 times 64
        kp[page, 0, slot, 0] = 7 if sign > 0 else 2        # 6, 1
        ks, vs = np.full((W, 1, 64, 2), 133, np.uint8), np.full((W, 1, 64, 2), 127, np.uint8)
        if way == "beyond":
            vp[page, 0, slot ^ 1, 0] = 0x77
            vs[page, 0, slot ^ 1, 0] = 150
        want = dev(O.values(vp[page, 0, slot], vs[page, 0, slot])).to(F16)
        for e in range(10, 41):
            for m in (1.0, 1.13, 1.37, 1.71):
                got = run(q, (kp, vp, ks, vs), table, [W * 64], sign * m * 2.0 ** e / 384, rows=rows)
                assert (got == want).all(), (at, e, m, got[0, :8].tolist(), want[:8].tolist())


# ------------------------------------------------------------------- values that bfloat16 does not hold

def cache(seed, W, H=1, dh=64):
    """Ordinary keys and values: [kp, vp, ks, vs], table [1][W]."""
    rng = np.random.default_rng(seed)
    (kp, ks), (vp, vs) = (O.quantise(rng.standard_normal((W, H, 64, dh))) for _ in "kv")
    return [kp, vp, ks, vs], rng.permutation(W).reshape(1, W).astype(np.int32)


def fill(pages, table, at, scale):
    """Every code under the scale bytes `scale` in the tokens `at` of the row: keys and values."""
    pages = [p.copy() for p in pages]
    for t in at:
        for i in (0, 1):
            pages[i][table[0, t // 64], :, t % 64] = np.arange(t, t + pages[i].shape[3]) * 7 % 256
            pages[i + 2][table[0, t // 64], :, t % 64] = scale
    return pages


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,S,W", PLANS)
def test_largest_scales_behind_the_limit_leave_a_query_alone(rows, S, W, dtype):
    """Tokens before a row's last one that no query sees, or only the last half of them, of scales whose larger
    codes are infinite in bfloat16: the others' results are the bits of a call that has 2^23 there."""
    n = W * 64
    pages, table = cache(W, W)
    q = torch.randn(S, 64, generator=torch.Generator().manual_seed(S)).to(dtype).cuda()
    for last in (n - 30, n - 64, n - 130 if S < 130 else n - 1):       # tokens that the last query sees
        half = S // 2
        for seen, at in ((S, range(last, n)), (half, range(last - S + half, n))):
            want = run(q, fill(pages, table, at, 150), table, [n], 0.125, [last - S], rows)
            o = O.attention(q.double().cpu().numpy()[None, :, None], *pages, table, [n], 0.125, 1, [last - S])[0]
            assert np.abs(want.double().cpu().numpy()[:seen] - o[0, :seen, 0]).max(initial=0) < 0.02
            for e in (253, 254, 255):
                print("attention_kv4 behind", rows, S, W, dtype, last, seen, e, flush=True)
                got = run(q, fill(pages, table, at, e), table, [n], 0.125, [last - S], rows)
                assert same(got[:seen], want[:seen])


@pytest.mark.parametrize("rows,S,W", PLANS)
def test_largest_bfloat16_values(rows, S, W):
    """bfloat16's largest numbers, appended: 2^128 as 4 bits have them.  Queries before them are as without,
    in the same block too; no result behind them is a number that is not near 2^128 times its share.  (Infinite
    or NaN it may be: a probability is up to 2^15 as two numbers of either sign, and both products pass
    2^128.)"""
    P, n = nv(), W * 64
    x = torch.randn(2, 1, n, 64, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    q = torch.randn(S, 64, generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    table = dev(np.random.default_rng(3).permutation(W).reshape(1, W).astype(np.int32))
    first, big = n - S // 2 - 5, torch.finfo(BF16).max
    outs = []
    for value in (2.0 ** 20, big):
        x[1, 0, first, 7] = value
        x[1, 0, first, 40] = -value
        d = P.nv_kv4_pages(W, 1, 64, "cuda")
        P.nv_op_kv4_append(x[0], x[1], d, table, dev(np.zeros(1, np.int32)))
        d = tuple(t.view(torch.uint8).cpu().numpy() for t in d)
        outs.append(run(q, d, table.cpu().numpy(), [n], 0.125, [n - S], rows))
    before = max(0, first - n + S)                                       # queries that end before it
    assert same(outs[0][:before], outs[1][:before]) and outs[0].isfinite().all()
    for c, sign in ((7, 1), (40, -1)):
        behind = sign * outs[1][before:, c].double().cpu()
        share = outs[0][before:, c].abs().double().cpu() / 2.0 ** 20     # of the token, about
        near = behind / 2.0 ** 128 / share
        assert near.numel() and ((near > 0.9) & (near < 1.1) | ~behind.isfinite()).all(), near


# ------------------------------------------------------------------------------- scales far apart

def bound(q, pages, table, n, scale, first, dtype):
    """(o, tol) [S][G][dh] of q [1][S][G][dh] over one row: a score is dh float32 additions and three products,
    the exponential 4 E |score| + 4 E, twice that for a probability (numerator and sum); its rounding 2^-11 of
    itself or 2^-34 of the query's largest where it is small, and then of the largest value of the channel
    that THIS query sees; n E for sums of n terms; one rounding of the result."""
    E, dh = 2.0 ** -23, q.shape[3]
    o, spread, size, most = O.attention(q, *pages, table, [n], scale, 1, [first])
    v = np.abs(O.row_of(pages[1], pages[3], table[0], n, 0)[0])
    last = np.clip(first + np.arange(q.shape[1]), -1, n - 1)
    seen = np.where(last[:, None] < 0, 0, np.maximum.accumulate(v)[last])[:, None]
    rel = 2 * (dh * E * size + 8 * E * most + 4 * E) + 2.0 ** -10 + n * E
    half = torch.finfo(dtype).eps / 2
    tol = rel * spread * (1 + half) + n * 2.0 ** -34 * (seen + np.abs(o)) + half * np.abs(o) \
        + (2.0 ** -25 if dtype == F16 else 0)
    return o[0], tol[0]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("S,G,N", [(9, 1, 1), (40, 1, 1), (300, 1, 1), (70, 4, 1), (120, 4, 96)])
def test_scales_far_apart_under_a_limit(S, G, N, dtype):
    """Values far above a query's own behind its limit leave its result as exact as without them, and values far
    below the largest keep their bits where only they are seen."""
    for dh in (64, 128):
        n, rng = 320, np.random.default_rng(S)
        for lo, hi in ((90, 138), (1, 120), (120, 130), (20, 160 if dtype == BF16 else 136)):
            pages, table = cache(2, 5, dh=dh)
            pages[3][:] = np.where(rng.random(pages[3].shape) < 0.02, lo, 126)
            pages[3][table[0, 1]] = lo
            pages[3][table[0, 3], :, 20:23] = hi        # tokens 212 to 214
            pages[3][table[0, 2], :, 7] = lo
            pages[3][table[0, 4], :, 8, -1] = hi
            if dtype == F16:                             # results within the type
                pages[1][table[0, 3], :, 20:23] &= 0x99
                pages[1][table[0, 4], :, 8] &= 0x99
            q = torch.randn(S, G * dh, generator=torch.Generator().manual_seed(S)).to(dtype).cuda()
            q64 = q.double().cpu().numpy().reshape(1, S, G, dh)
            for first in (n - S, 200 - S // 2, 211 - S):
                print("attention_kv4 far", S, G, N, dtype, dh, lo, hi, first, flush=True)
                got = run(q, pages, table, [n], dh ** -0.5, [first], N).double().cpu().numpy()
                o, tol = bound(q64, pages, table, n, dh ** -0.5, first, dtype)
                bad = ~(np.abs(got.reshape(o.shape) - o) <= tol)
                assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dh", [16, 32, 40, 64, 80, 128, 160])
def test_large_scores_of_any_head(dh, dtype):
    """The largest of scores of 2^23 to 2^38 under tiles of 16, 64 and 128, in ordinary pages and in pages that
    16 bits do not hold."""
    W, rng = 6, np.random.default_rng(dh)
    table = rng.permutation(W).reshape(1, W).astype(np.int32)
    nb = -(-dh // 32)
    for rows, S in ((1, 3), (1, 300), (300, 300)):
        print("attention_kv4 large scores", rows, S, dh, dtype, flush=True)
        q = torch.zeros(S, dh, dtype=dtype, device="cuda")
        q[:, dh - 1] = 1 + torch.arange(S, device="cuda") % 61 / 64
        for at, way in ((70, 0), (W * 64 - 1, 0), (130, 1)):
            page, slot = table[0, at // 64], at % 64
            kp = np.zeros((W, 1, 64, dh // 2), np.uint8)
            kp[..., -1] = rng.integers(4, 7, (W, 1, 64)) << 4
            kp[page, 0, slot, -1] = 7 << 4
            vp = rng.integers(0, 256, (W, 1, 64, dh // 2)).astype(np.uint8)
            ks, vs = np.full((W, 1, 64, nb), 133, np.uint8), np.full((W, 1, 64, nb), 127, np.uint8)
            if way:
                vp[page, 0, slot ^ 1, 0], vs[page, 0, slot ^ 1, 0] = 0x77, 150
            want = dev(O.values(vp[page, 0, slot], vs[page, 0, slot])).to(dtype)
            for e in range(23, 39):
                got = run(q, (kp, vp, ks, vs), table, [W * 64], 1.37 * 2.0 ** e / 384, rows=rows)
                assert (got == want).all(), (at, e)
