"""Attention over the 4-bit cache where the work is shared out: one sequence over many
blocks of threads, long lists of short sequences, pools beyond 32-bit offsets. The bounds are
those of test_gpu_cache_attend."""
import math

import numpy as np
import pytest
import torch

from cache_helpers import f64, ints, make, ok, rows
from paper_2607_20940_gb300 import msf
from test_gpu_cache_attend import check, fill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group,queries", [(1, 1), (4, 5), (8, 3), (2, 15), (1, 33), (4, 25), (1, 128), (2, 100), (1, 300)])
def test_one_long_sequence(D, group, queries):
    """Its steps go to most of the grid, so an item has tens of pieces (and 17 to 24 rows one block)."""
    lens = [9001]
    c = make(kv_heads=1, head_dim=D, page_tokens=64, sequences=1, sequence_pages=160, pages=160)
    kh, vh = fill(c, lens, 21)
    q = rows((1, queries, group, D), 22)
    first = check(c, kh, vh, lens, q, True)
    base = rows(q.shape, 23)
    base_lse = torch.randn(1, group, queries, generator=torch.Generator().manual_seed(24)).cuda() * 2 + 8
    base_lse[0, 0, 0] = -math.inf
    check(c, kh, vh, lens, q, True, base, base_lse)
    for _ in range(3):  # whichever block ends last
        again = torch.empty_like(q), torch.empty_like(base_lse)
        c.attend(0, q, *again, causal=True)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group,queries", [(3, 6), (1, 24), (2, 17)])
def test_a_few_sequences_of_any_length(D, group, queries):
    lens = [2500, 0, 31, 5000, 16, 1]
    c = make(kv_heads=2, head_dim=D, page_tokens=32, sequences=6, sequence_pages=160, pages=400)
    kh, vh = fill(c, lens, 31)
    for causal in (False, True):
        check(c, kh, vh, lens, rows((6, queries, 2 * group, D), 32), causal)


@pytest.mark.parametrize("group,queries", [(1, 1), (2, 10), (1, 40), (1, 260)])
def test_lists_longer_than_a_block(group, queries):
    lens = [5, 0, 140, 33, 64]
    c = make(kv_heads=1, head_dim=64, sequences=5, pages=30)
    kh, vh = fill(c, lens, 41)
    n = 1100 if queries < 100 else 530
    seqs = [(7 * i + i // 9) % 5 for i in range(n)]
    check(c, kh, vh, lens, rows((n, queries, group, 64), 42), True, seqs=seqs)


def test_offsets_past_32_bits():
    """A pool of 4.8 GB whose low pages are taken: appended, read back, attended, copied, moved."""
    P, low = 128, 31000
    c = make(kv_heads=8, head_dim=128, page_tokens=P, sequences=3, sequence_pages=low, pages=32700)
    assert low * c.info.page_bytes > 2 ** 32
    c.grow(ints([0]), ints([low * P]))
    n = 3 * P + 5
    k, v = rows((1, n, 8, 128), 51), rows((1, n, 8, 128), 52)
    c.grow(ints([1]), ints([n]))
    c.write(0, k, v, ints([1]))
    ok(c)
    assert int(c.table[1, 0]) == low
    k0, v0 = torch.empty_like(k), torch.empty_like(v)
    c.read(0, k0, v0, ints([1]))
    kh, vh = (np.concatenate([np.zeros_like(f64(x)), f64(x)]) for x in (k0, v0))
    # (a code is at most 1 off where the largest is 6, and the scale 2^-4 of itself: less than a quarter)
    assert (np.abs(kh[1] - f64(k)[0]) <= np.abs(f64(k)[0]).reshape(n, 8, 8, 16).max(-1).repeat(16, -1) / 4).all()
    for queries in (1, 40):
        q = rows((1, queries, 16, 128), 53)
        want = check(c, kh, vh, [0, n], q, seqs=[1])
        c.fork(ints([1]), ints([2]), copy=True)
        check(c, np.concatenate([kh, kh[1:]]), np.concatenate([vh, vh[1:]]), [0, n, n], q, seqs=[2])
    c.truncate(ints([0]))
    c.compact()
    ok(c)
    assert int(c.table[1:, :4].max()) == 7
    out, lse = torch.empty_like(q), torch.empty_like(want[1])
    for s in (1, 2):
        c.attend(0, q, out, lse, seqs=ints([s]))
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_a_wait_that_gave_up_is_reported():
    """The status word of a kernel whose bounded wait ran out, planted from the host."""
    c = make()
    c.bound_state[:4].view(torch.int32).fill_(1)
    assert c.device_status() == msf.MSF_ERR_TIMEOUT
    lens = [40, 0, 3, 100]
    kh, vh = fill(c, lens, 61)
    check(c, kh, vh, lens, rows((4, 2, 2, 64), 62))


@pytest.mark.parametrize("group,queries", [(1, 257), (3, 100), (2, 192), (4, 128), (1, 513), (5, 140), (1, 1100)])
@pytest.mark.parametrize("causal", [False, True])
def test_blocks_of_two(group, queries, causal):
    """Over sequences that may hold 1536 tokens or more, more than 256 rows go to pairs of blocks of threads."""
    lens = [0, 1, 15, 17, 64, 65, 113, 128, 129, 500, 1600]
    c = make(kv_heads=2, head_dim=128, page_tokens=32, sequences=len(lens), sequence_pages=50, pages=120)
    kh, vh = fill(c, lens, 71)
    q = rows((len(lens), queries, 2 * group, 128), 72)
    check(c, kh, vh, lens, q, causal)
    seqs = [10, 3, 10, 0]
    base = rows((4, *q.shape[1:]), 73)
    base_lse = torch.randn(4, 2 * group, queries, generator=torch.Generator().manual_seed(74)).cuda() * 2 + 4
    base_lse[1, 0, 0] = base_lse[3, 1, 2] = -math.inf
    wide = torch.zeros(4, queries + 3, 2 * group, 128 + 8, dtype=torch.bfloat16, device="cuda")
    strided = wide[:, 1:1 + queries, :, 8:]
    strided.copy_(q[:4])
    first = check(c, kh, vh, lens, strided, causal, base, base_lse, scale=0.2, seqs=seqs)
    for _ in range(2):
        again = torch.empty_like(base), torch.empty_like(base_lse)
        c.attend(0, strided, *again, base, base_lse, ints(seqs), causal, 0.2)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_blocks_of_two_with_scores_far_apart():
    """Every 40th key is far ahead, so maxima move late and by much."""
    n, queries = 1700, 300
    c = make(kv_heads=1, head_dim=128, page_tokens=64, sequences=1, sequence_pages=32, pages=32)
    k, v = rows((1, n, 1, 128), 81, 0.2), rows((1, n, 1, 128), 82)
    k[:, ::40] *= torch.linspace(1, 30, len(range(0, n, 40)), device="cuda", dtype=torch.bfloat16)[None, :, None, None]
    c.grow(None, ints([n]))
    c.write(0, k, v)
    ok(c)
    k0, v0 = torch.empty_like(k), torch.empty_like(v)
    c.read(0, k0, v0)
    for causal in (False, True):
        check(c, f64(k0), f64(v0), [n], rows((1, queries, 1, 128), 83, 3.0), causal, floor=2.0 ** -30)
