"""What the GPU tests of values far apart rest on, without a GPU: that a kernel which loses a page, or
rounds to fewer bits than stated, exceeds their bounds."""
import numpy as np
import pytest

import ops8_values as V


def exceeds(q, pages, other, table, lens, scale, qpos=None):
    """Whether the exact outputs over `other` pages would fail the bound of those over `pages`."""
    o, tol = V.attention(q, pages, table, lens, scale, qpos)
    wrong, _ = V.attention(q, other, table, lens, scale, qpos)
    return np.abs(wrong - o) > 4 * tol


@pytest.mark.parametrize("order", sorted(V.ORDERS))
@pytest.mark.parametrize("d", V.DISTANCES)
def test_a_lost_page_far_below_the_largest_exceeds_the_bound(d, order):
    q = V.queries(3, 1, 64)
    pages, table = V.far_cache(d, order)
    n = 64 * table.shape[1]
    for lens, qpos in (([n], None), ([n - 2], [n - 5])):
        for j, below in enumerate(V.ORDERS[order]):
            lost = [p.copy() for p in pages]
            lost[1][table[0, j]] = 0
            bad = exceeds(q, pages, lost, table, lens, 0.125, qpos)[..., :32] if below else \
                exceeds(q, pages, lost, table, lens, 0.125, qpos)[..., 32:]
            assert bad.any((0, 2, 3)).all() and bad.mean() > 0.5, (d, order, j)
            if below:  # a factor of two in its size, too
                lost = [p.copy() for p in pages]
                lost[3][table[0, j]] += 1
                assert exceeds(q, pages, lost, table, lens, 0.125, qpos)[..., :32].mean() > 0.5


def rounded_probabilities(q, pages, table, n, scale, top):
    """Attention whose largest probability is 2^top when they are rounded to float16, their sum exact."""
    from oracle import ops8 as O
    k, _ = O.read_cache(pages[0], pages[2], table[0], n, 0, False)
    v, _ = O.read_cache(pages[1], pages[3], table[0], n, 0, True)
    a = q[0, :, 0] @ k.T * scale
    p = np.exp(a - a.max(1, keepdims=True)) * 2.0 ** top
    return (p.astype(np.float16).astype(np.float64) @ v / p.sum(1, keepdims=True))[None, :, None]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits,spread", V.TAILS)
def test_probabilities_below_1_exceed_the_bound_of_a_tail(bits, spread, dtype):
    """... and from 2^9 on they keep it."""
    q, pages, table, n, scale = V.tail_cache(3, 0, bits, spread)
    o, tol = V.attention(q, pages, table, [n], scale, dtype=dtype)
    err = lambda top: (np.abs(rounded_probabilities(q, pages, table, n, scale, top) - o) / tol).max()
    assert err(9) <= 1 and err(15) <= 1
    assert err(0) > 1 or bits < 24
