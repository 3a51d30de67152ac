"""Pins of the 4-bit cache's oracle (CPU): the format by exhaustion and by hand, the
attention against torch's, the page model's invariants."""
import random

import numpy as np
import pytest
import torch

from oracle import cache as oc


def test_scales_are_e4m3():
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.sort(t), oc.E4M3)


def test_codes_are_the_nearest_values():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((64, 32)) * np.exp2(rng.integers(-8, 8, (64, 1)))
    v, code, s = oc.quantise(x)
    every = oc.GRID * s[..., None, None]  # [64, 2, 1, 8]
    best = np.abs(np.abs(x).reshape(64, 2, 16, 1) - every).min(-1)
    assert np.allclose(np.abs(x - v).reshape(64, 2, 16), best, rtol=0, atol=1e-12)
    want = np.abs(x).reshape(64, 2, 16).max(-1) / 6
    best = np.abs(want[..., None] - oc.E4M3[1:]).min(-1)  # never 0
    assert np.array_equal(np.abs(want - s), best)


def test_by_hand():
    x = np.zeros(16)
    # amax 6, scale 1; ties to the even code: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    x[:9] = [6, 0.25, 0.75, 1.25, 1.75, -2.5, 3.5, -5, 0.26]
    v, _, s = oc.quantise(x)
    assert s[0] == 1 and list(v[:9]) == [6, 0, 1, 1, 2, -2, 4, -4, 0.5]
    # a scale that rounds down saturates: amax 6 * 17/16 -> tie of 1 and 1.125, even mantissa 1
    x[:] = 0
    x[0] = 6 * 17 / 16
    v, _, s = oc.quantise(x)
    assert s[0] == 1 and v[0] == 6
    # the smallest scale, and far above the largest
    x[0] = 2.0 ** -20
    assert oc.quantise(x)[2][0] == 2.0 ** -9 and oc.quantise(x)[0][0] == 0
    x[0] = 1e30
    assert oc.quantise(x)[2][0] == 448 and oc.quantise(x)[0][0] == 2688
    assert oc.quantise(x * 2.0 ** -5, -5)[0][0] == 2688 * 2.0 ** -5
    x[:3] = [np.nan, -np.inf, 1.0]
    assert list(oc.quantise(x)[0][:3]) == [0, -2688, 0]


def test_values_of_the_cache_stay():
    """What was read out and goes in again is the same, where the largest code is in its block."""
    rng = np.random.default_rng(2)
    code = rng.integers(0, 8, (50, 16))
    code[:, 3] = 7
    v = oc.GRID[code] * np.where(rng.random((50, 16)) < 0.5, -1, 1) * rng.choice(oc.E4M3[1:], (50, 1))
    assert np.array_equal(oc.quantise(v)[0], v)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,nq", [(7, 1), (9, 4), (3, 5)])
def test_attend_matches_torch(n, nq, causal):
    rng = np.random.default_rng(n)
    q, k, v = rng.standard_normal((nq, 2, 16)), rng.standard_normal((n, 16)), rng.standard_normal((n, 16))
    out, lse, _, _ = oc.attend(q, k, v, causal)
    mask = torch.ones(nq, n, dtype=torch.bool)
    if causal:
        mask = mask.tril(n - nq)
    for h in range(2):
        want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x) for x in (q[:, h], k, v)),
                                                                attn_mask=mask).numpy()
        seen = mask.any(1).numpy()
        assert np.allclose(out[seen, h], want[seen]) and not out[~seen].any()
        assert np.all(np.isneginf(lse[h][~seen]))
    # two halves, joined, are the whole
    a = oc.attend(q, k[:2], v[:2])
    b = oc.attend(q, k[2:], v[2:], base=a[0], base_lse=a[1])
    whole = oc.attend(q, k, v)
    assert np.allclose(b[0], whole[0]) and np.allclose(b[1], whole[1])


def test_pages_hold_together():
    rng = random.Random(5)
    for _ in range(30):
        P, S = rng.choice([16, 32]), 6
        m = oc.Pages(40, S, P, 12)
        for _ in range(40):
            before = (m.table_array().copy(), list(m.lengths))
            op = rng.randrange(4)
            some = rng.sample(range(S), rng.randint(1, S))
            try:
                if op == 0:
                    m.grow(some, [rng.randint(0, 3 * P) for _ in some])
                elif op == 1:
                    m.fork([rng.randrange(S) for _ in some], some, [rng.randint(0, 100) for _ in some], rng.random() < 0.5)
                elif op == 2:
                    m.truncate(some, [rng.randint(0, 60) for _ in some])
                else:
                    m.compact()
                    used = [p for p, r in enumerate(m.refs()) if r]
                    assert used == list(range(len(used)))
            except oc.Full:
                assert np.array_equal(before[0], m.table_array()) and before[1] == m.lengths
            assert all(len(row) == m.need(n) for row, n in zip(m.table, m.lengths))
            assert all(len(set(row)) == len(row) for row in m.table)
