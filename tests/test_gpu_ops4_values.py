"""Attention over the 4-bit cache where scores are far from one another in size, against the value that the
definition picks."""
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
