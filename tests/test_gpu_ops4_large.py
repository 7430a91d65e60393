"""The rotation and the 4-bit cache at sizes from which on their kernels work in another way: reads of two units
a lane, rotations whose tokens share a workgroup, attention of more workgroups than are resident."""
import numpy as np
import pytest
import torch

from oracle import ops4 as O
from test_gpu_ops4 import BF16, E, F16, F32, a_cache, check_attention, dev, i32, np64, nv, rand, spoil, u

pytestmark = pytest.mark.gpu


# -------------------------------------------------------------------------------------- read

@pytest.fixture(scope="module")
def held():
    """A cache of any codes and scales, what is asked of it, and what the oracle reads: 2.15 million units of
    eight channels, each row's no multiple of two units of a workgroup."""
    R, T, H, dh, W = 7, 4801, 8, 64, 80
    rng = np.random.default_rng(0)
    P = R * W + 1
    pages = [rng.integers(0, 256, (P, H, 64, dh // 2)).astype(np.uint8) for _ in "kv"] + \
        [rng.integers(100, 150, (P, H, 64, dh // 32)).astype(np.uint8) for _ in "kv"]
    pages[2][rng.random(pages[2].shape) < 0.01] = 255
    pages[3][rng.random(pages[3].shape) < 0.01] = 0
    table = rng.permutation(P)[:R * W].reshape(R, W).astype(np.int32)
    table[1, 30], table[2, 0], table[3, W - 1] = -1, P, 10 ** 9
    pos, count = np.array([0, 17, 319, 330, 64, 1, -4]), np.array([T, T, T, T, 2000, T - 1, T])
    want = [O.read(c, s, table, pos, T, count) for c, s in ((pages[0], pages[2]), (pages[1], pages[3]))]
    return pages, table, pos, count, T, want


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("at,extra", [(0, 0), (16, 24), (3, 6)])
def test_read_of_many_tokens(held, at, extra, dtype):
    """Rows of their own, rows inside a larger buffer, rows off 16 bytes: ragged counts, holes, a row of
    nothing, tokens past the table."""
    pages, table, pos, count, T, want = held
    R, cols = table.shape[0], want[0].shape[2]
    print("read4", at, extra, dtype, flush=True)
    big = [torch.full((R, T + 1, cols + extra), 5.0, dtype=dtype, device="cuda") for _ in "kv"]
    out = tuple(b[:, :T, at:at + cols] for b in big)
    nv().nv_op_kv4_read(tuple(dev(p) for p in pages), i32(table), i32(pos), T, i32(count), dtype, out=out)
    for b, g, w in zip(big, out, want):
        w = torch.from_numpy(w).to(dtype).cuda()
        assert torch.equal(g.nan_to_num(7, 8, 9), w.nan_to_num(7, 8, 9))
        assert (b[:, T] == 5).all() and (b[:, :, :at] == 5).all() and (b[:, :, at + cols:] == 5).all()


# -------------------------------------------------------------------------------------- rope

# rows, tokens, query heads, key heads, dh, axes: 5, 10 and 40 steps of a workgroup's heads, then 3 and 2; tokens
# that share a workgroup 4, 4, 1, 13 and 16, rows that end inside one
ROPES = [(3, 1401, 14, 6, 128, (48, 48, 32), (44, 42, 42)), (3, 1401, 32, 8, 128, (128,), (2, 30, 32, 64)),
         (2, 2101, 130, 30, 128, (64, 64), (44, 42, 42)), (5, 3301, 12, 8, 64, (16, 48), (22, 20)),
         (1, 16411, 8, 2, 40, (32,), (14, 26))]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("pairs", ["next", "halves of 16", "any halves"])
@pytest.mark.parametrize("R,S,Hq,H,dh,by16,uneven", ROPES)
def test_rope_of_many_tokens(R, S, Hq, H, dh, by16, uneven, pairs, dtype):
    """Every bit as from calls of few tokens, and a sample of tokens against the oracle."""
    axes, halves = by16 if pairs == "halves of 16" else uneven, pairs != "next"
    print("rope", R, S, Hq, H, dh, axes, halves, dtype, flush=True)
    P, rng = nv(), np.random.default_rng(S)
    qkv = rand(S, R, S, (Hq + 2 * H) * dh, dtype=dtype)
    q, k = qkv[..., :Hq * dh], qkv[..., Hq * dh:(Hq + H) * dh]
    places = rng.integers(0, 200_000, (R, S, len(axes)))
    pos, f = i32(places), P.nv_rope_freqs(axes)
    w = [1 + 0.2 * rand(i, dh) for i in (1, 2)]
    got = P.nv_op_qk_rope(q, k, dh, pos, axes, f, *w, halves=halves)
    for r in range(R):
        for a in range(0, S, 500):
            b = min(S, a + 500)
            few = P.nv_op_qk_rope(q[r:r + 1, a:b], k[r:r + 1, a:b], dh, pos[r:r + 1, a:b], axes, f, *w,
                                  halves=halves)
            for g, x in zip(got, few):
                assert torch.equal(g[r, a:b], x[0]), (r, a)
    at = np.unique(np.concatenate([rng.integers(0, S, 40), [0, S - 1]]))
    for x, y, wt in ((q, got[0], w[0]), (k, got[1], w[1])):
        y = np64(y[:, at])
        want, size = O.rope(np64(x[:, at]).reshape(R, len(at), -1, dh), places[:, at], axes, np64(f), np64(wt),
                            1e-6, halves)
        tol = 30 * E * size + u(dtype) * np.abs(want) + (2.0 ** -25 if dtype == F16 else 0)
        assert (np.abs(y.reshape(want.shape) - want) <= tol).all()
    P.nv_op_qk_rope(q, k, dh, pos, axes, f, *w, halves=halves, out=(q, k))  # in place
    assert torch.equal(q, got[0]) and torch.equal(k, got[1])


# --------------------------------------------------------------------------------- attention

@pytest.mark.parametrize("R,S,H,G,dh,W", [(4, 544, 8, 4, 40, 10), (10, 300, 8, 4, 64, 6), (8, 600, 8, 2, 160, 10)])
def test_causal_tiles_of_more_workgroups_than_are_resident(R, S, H, G, dh, W):
    """Tiles of 128 queries, longest first: rows of differing length, one with a hole."""
    print("attention_kv4 causal", R, S, H, G, dh, W, flush=True)
    pages, table = a_cache(S, R, W, H, dh)
    lens = [W * 64 - 37 * r for r in range(R)]
    spoil(pages, table, lens)
    table[1, 1] = -1
    q = rand(S, R, S, H * G * dh, dtype=BF16)
    check_attention(q, pages, table, lens, dh ** -0.5, H, [n - S for n in lens])
