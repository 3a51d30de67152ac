"""Attention over the 4-bit cache against the same attention in 64 bits over the values held.

Bounds, from the arithmetic: the output's rounding to bf16 is 2^-9 of it; probabilities may
be rounded to 11 bits on the way, 2^-11 of sum p |v| (A below); a score of D products summed in
fp32 is off by at most D 2^-24 of scale sum |q k| (B), which changes probabilities by that
share, twice with the sum. Twice all of it is allowed. Probabilities below 2^-19 of a row's
largest are multiples of 2^-29 of it (f16's smallest), so each may be 2^-30 off: that counts
where keys' scores lie far apart (`floor`; the fp32 form has none). The log-sum-exp has the scores' error
and 2^-20 of one for exponentials and sums."""
import math

import numpy as np
import pytest
import torch

from cache_helpers import f64, ints, make, ok, rows
from oracle import cache as oc
from paper_2607_20940_gb300 import msf

pytestmark = pytest.mark.gpu


def fill(c, lens, seed, k_std=1.0):
    """Sequences of these lengths; the values held [S, longest, Hk, D] in 64 bits."""
    H, D, n = c.desc.kv_heads, c.desc.head_dim, max(1, max(lens))
    k, v = rows((len(lens), n, H, D), seed, k_std), rows((len(lens), n, H, D), seed + 1)
    k = k * 2.0 ** c.desc.k_exponent
    v = v * 2.0 ** c.desc.v_exponent
    step = -(-n // 3)  # in turns, so that pages of different sequences alternate
    for at in range(0, n, step):
        m = min(step, n - at)
        counts = ints([min(m, max(0, x - at)) for x in lens])
        c.grow(None, counts)
        c.write(0, k[:, at:at + m], v[:, at:at + m], None, counts)
    ok(c)
    return oc.quantise(f64(k), c.desc.k_exponent)[0], oc.quantise(f64(v), c.desc.v_exponent)[0]


def check(c, kh, vh, lens, q, causal=False, base=None, base_lse=None, scale=None, seqs=None, out=None, lse=None,
          simt=False, floor=0.0):
    D, r = c.desc.head_dim, q.shape[2] // c.desc.kv_heads
    n, nq = q.shape[:2]
    if out is None:
        out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    if lse is None:
        lse = torch.full((n, q.shape[2], nq), 9.0, device="cuda")
    b = f64(base) if base is not None else None
    bl = f64(base_lse) if base is not None else None
    c.attend(0, q, out, lse, base, base_lse, ints(seqs), causal, scale or 0.0, simt=simt)
    ok(c)
    got, got_lse, qq = f64(out), f64(lse), f64(q)
    for i in range(n):
        s = seqs[i] if seqs is not None else i
        for h in range(c.desc.kv_heads):
            hs = slice(h * r, h * r + r)
            want, want_lse, A, B = oc.attend(qq[i][:, hs], kh[s, :lens[s], h], vh[s, :lens[s], h], causal, scale,
                                             None if b is None else b[i][:, hs], None if b is None else bl[i, hs])
            share = D * 2.0 ** -24 * B
            bound = 2 * (2.0 ** -9 * np.abs(want) + (2.0 ** -11 + 2 * share) * A) + 1e-30
            bound += 2 * floor * np.abs(vh[s, :lens[s], h]).sum(0)
            assert (np.abs(got[i][:, hs] - want) <= bound).all(), (i, h, np.max(np.abs(got[i][:, hs] - want) / bound))
            empty = np.isneginf(want_lse)
            assert np.array_equal(empty, np.isneginf(got_lse[i, hs]))
            e = np.abs(got_lse[i, hs][~empty] - want_lse[~empty])
            assert (e <= 2 * share + 2.0 ** -20 * (1 + np.abs(want_lse[~empty]))).all(), e.max()
    return out, lse


# rows of one key head: group * queries
SHAPES = [(1, 1), (4, 1), (8, 1), (3, 3), (16, 1), (1, 16), (1, 17), (5, 7), (2, 40), (1, 129), (4, 70), (1, 300)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group,queries", SHAPES)
@pytest.mark.parametrize("causal", [False, True])
def test_shapes(D, group, queries, causal):
    lens = [0, 1, 15, 16, 17, 64, 127, 128, 129, 383, 500]
    c = make(kv_heads=2, head_dim=D, sequences=len(lens), sequence_pages=32, pages=100)
    kh, vh = fill(c, lens, 3)
    check(c, kh, vh, lens, rows((len(lens), queries, 2 * group, D), 5), causal)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("queries", [1, 60])
def test_pages_that_end_inside_a_tile(P, queries):
    lens = [P, P + 1, 3 * P - 1, 700, 2 * P]
    c = make(kv_heads=1, head_dim=128, page_tokens=P, sequences=5, sequence_pages=-(-700 // P), pages=3000 // P + 20)
    kh, vh = fill(c, lens, 4)
    check(c, kh, vh, lens, rows((5, queries, 2, 128), 6), queries > 1)


@pytest.mark.parametrize("group,queries", [(1, 1), (4, 2), (1, 50)])
@pytest.mark.parametrize("causal", [False, True])
def test_joined_with_another_attention(group, queries, causal):
    lens = [0, 3, 200, 45]
    c = make(kv_heads=2, head_dim=128, sequences=4, pages=60)
    kh, vh = fill(c, lens, 5)
    q = rows((4, queries, 2 * group, 128), 7)
    base = rows(q.shape, 8)
    base_lse = torch.randn(4, 2 * group, queries, generator=torch.Generator().manual_seed(9)).cuda() * 3 + 3
    base_lse[2, 0, 0] = base_lse[0, 1, 0] = -math.inf  # rows that the other attention left empty
    base[0, 0, 1] = float("nan")  # and what stands there does not count
    clean = base.clone()
    clean[0, 0, 1] = 0
    out, lse = torch.empty_like(q), torch.empty_like(base_lse)
    c.attend(0, q, out, lse, base, base_lse, causal=causal)
    want = check(c, kh, vh, lens, q, causal, clean, base_lse)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    # in place
    x, y = base.clone(), base_lse.clone()
    c.attend(0, q, x, y, x, y, causal=causal)
    assert torch.equal(x, out) and torch.equal(y, lse)
    x = base.clone()
    c.attend(0, q, x, None, x, base_lse, causal=causal)
    assert torch.equal(x, out)


def test_strides_lists_and_scales():
    lens = [33, 0, 260]
    c = make(kv_heads=2, head_dim=64, sequences=3, pages=40, sequence_pages=20, k_exponent=3, v_exponent=-5)
    kh, vh = fill(c, lens, 6)
    for queries in (1, 37):
        seqs = [2, 0, 2, 1]
        wide = rows((4, queries + 5, 8, 72), 7)
        q = wide[:, 2:2 + queries, 1:7, 8:].contiguous()
        strided = wide[:, 2:2 + queries, 1:7, 8:]
        hold = torch.full((4, 9, queries + 3, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        out = hold[:, 2:8, 1:queries + 1].transpose(1, 2)  # heads outside of queries
        lse_hold = torch.full((4, 8, queries + 2), 5.0, device="cuda")
        lse = lse_hold[:, 1:7, 1:queries + 1]
        check(c, kh, vh, lens, strided, True, scale=0.05, seqs=seqs, out=out, lse=lse)
        again = torch.empty_like(q)
        c.attend(0, q, again, seqs=ints(seqs), causal=True, softmax_scale=0.05)
        assert torch.equal(again, out)
        out.fill_(5.0)
        lse.fill_(5.0)
        assert (hold == 5.0).all() and (lse_hold == 5.0).all()


@pytest.mark.parametrize("simt", [True, False])
@pytest.mark.parametrize("group,queries", [(4, 1), (1, 64)])
def test_scores_far_apart(group, queries, simt):
    """Rows whose largest score comes late, is huge, or stands alone among keys that do not count."""
    c = make(kv_heads=1, head_dim=128, sequences=3, pages=200, sequence_pages=64)
    lens = [900, 1000, 64]
    kh, vh = fill(c, lens, 7, k_std=8.0)
    q = rows((3, queries, group, 128), 8, 12.0)
    q[1, :, 0] *= 1e-3
    q[0, -1, -1] = 0
    form = dict(simt=simt, floor=0.0 if simt else 2.0 ** -30)
    check(c, kh, vh, lens, q, **form)
    check(c, kh, vh, lens, q * 2.0 ** -60, scale=2.0 ** 50, **form)
    check(c, kh, vh, lens, (q * 2.0 ** 40), scale=2.0 ** -41, **form)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("group,queries", [(1, 1), (3, 5), (2, 40)])
def test_fp32_form(group, queries, causal):
    lens = [0, 1, 17, 300]
    for D in (64, 128):
        c = make(kv_heads=2, head_dim=D, sequences=4, sequence_pages=32, pages=60)
        kh, vh = fill(c, lens, 20)
        q = rows((4, queries, 2 * group, D), 21)
        check(c, kh, vh, lens, q, causal, simt=True)
        base, base_lse = rows(q.shape, 22), torch.ones(4, 2 * group, queries, device="cuda")
        check(c, kh, vh, lens, q, causal, base, base_lse, simt=True)


@pytest.mark.parametrize("group,queries", [(8, 1), (1, 1), (1, 200), (2, 33)])
def test_long_and_ragged(group, queries):
    lens = [5000, 1, 0, 2049, 4096]
    c = make(kv_heads=1, head_dim=128, page_tokens=32, sequences=5, sequence_pages=160, pages=400)
    kh, vh = fill(c, lens, 9)
    check(c, kh, vh, lens, rows((5, queries, group, 128), 10), queries > 1)


def test_the_same_bits_again():
    c = make(kv_heads=2, head_dim=128, page_tokens=32, sequences=3, sequence_pages=160, pages=400)
    fill(c, [5000, 300, 1777], 11)
    for group, queries in ((4, 1), (1, 150)):
        q = rows((3, queries, 2 * group, 128), 12)
        a, la = torch.empty_like(q), torch.empty(3, 2 * group, queries, device="cuda")
        c.attend(0, q, a, la, causal=True)
        for _ in range(5):
            b, lb = torch.empty_like(q), torch.empty_like(la)
            c.attend(0, q, b, lb, causal=True)
            assert torch.equal(a, b) and torch.equal(la, lb)


def test_forked_copied_and_moved_sequences_answer_alike():
    c = make(layers=1, kv_heads=2, head_dim=64, sequences=6, sequence_pages=16, pages=80)
    kh, vh = fill(c, [100, 37, 0, 0, 0, 0], 13)
    c.fork(ints([0, 1]), ints([2, 3]))
    c.fork(ints([0]), ints([4]), ints([50]), copy=True)
    ok(c)
    q = rows((1, 4, 4, 64), 14)
    at = lambda s: _attend(c, q, s)  # noqa: E731
    whole = {s: at(s) for s in range(5)}
    assert torch.equal(whole[0], whole[2]) and torch.equal(whole[1], whole[3])
    # the first sequence ends, the rest moves down, a fork goes on alone
    c.truncate(ints([0]))
    c.compact()
    ok(c)
    for s in (1, 2, 3, 4):
        assert torch.equal(whole[s], at(s))
    x = rows((1, 1, 2, 64), 15)
    c.grow(ints([3]), None, 1)
    c.write(0, x, x, ints([3]))
    ok(c)
    assert torch.equal(whole[1], at(1)) and not torch.equal(whole[3], at(3))
    k2, v2 = oc.quantise(f64(x))[0], oc.quantise(f64(x))[0]
    kk = np.concatenate([kh[1:2, :37], k2], 1)
    vv = np.concatenate([vh[1:2, :37], v2], 1)
    check(c, np.repeat(kk, 4, 0), np.repeat(vv, 4, 0), [38] * 4, q, seqs=[3])


def _attend(c, q, s):
    out = torch.empty_like(q)
    c.attend(0, q, out, seqs=ints([s]))
    ok(c)
    return out


def test_another_stream_and_graph():
    lens = [70, 300]
    c = make(kv_heads=1, head_dim=128, sequences=2, pages=60, sequence_pages=24)
    kh, vh = fill(c, lens, 16)
    q = rows((2, 3, 4, 128), 17)
    want, want_lse = check(c, kh, vh, lens, q, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = torch.empty_like(q), torch.empty_like(want_lse)
    c.attend(0, q, out, lse, causal=True, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    g = torch.cuda.CUDAGraph()
    out.zero_()
    x = rows((2, 1, 1, 128), 18)
    with torch.cuda.graph(g):  # a decoding step: the same graph at any length
        c.grow(tokens=1)
        c.write(0, x, x)
        c.attend(0, q, out, lse, causal=True)
    held = oc.quantise(f64(x))[0]
    kk, vv = kh[:, :300].copy(), vh[:, :300].copy()
    kk, vv = (np.concatenate([y, np.zeros((2, 40, 1, 128))], 1) for y in (kk, vv))
    n = list(lens)
    for _ in range(20):
        g.replay()
        for s in range(2):
            kk[s, n[s]], vv[s, n[s]] = held[s, 0], held[s, 0]
            n[s] += 1
    ok(c)
    again = out.clone()
    want, _ = check(c, kk, vv, n, q, True)
    assert torch.equal(again, want)


@pytest.mark.parametrize("queries", [1, 5, 140])
def test_newest_tokens_that_are_not_seen(queries):
    lens = [40, 7, 0, 300]
    c = make(kv_heads=2, head_dim=64, sequences=4, pages=60, sequence_pages=24)
    kh, vh = fill(c, lens, 30)
    q = rows((4, queries, 4, 64), 31)
    for causal in (False, True):
        for simt in (False, True):
            out, lse = torch.empty_like(q), torch.empty(4, 4, queries, device="cuda")
            c.attend(0, q, out, lse, causal=causal, skip=16, simt=simt)
            c.truncate(None, ints([max(0, n - 16) for n in lens]))
            want, want_lse = check(c, kh, vh, [max(0, n - 16) for n in lens], q, causal, simt=simt)
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
            c.grow(None, ints([n - max(0, n - 16) for n in lens]))  # the same pages again


def test_refusals():
    c = make(kv_heads=2, head_dim=64)
    q = rows((4, 3, 4, 64), 1)
    out, lse = torch.empty_like(q), torch.empty(4, 4, 3, device="cuda")
    bad = [lambda: c.attend(1, q, out), lambda: c.attend(0, q[:, :, :3], out[:, :, :3]),
           lambda: c.attend(0, q, out, lse, base_out=q), lambda: c.attend(0, q, out, lse, base_lse=lse),
           lambda: c.attend(0, q, out, softmax_scale=-1.0), lambda: c.attend(0, q, out, softmax_scale=math.nan), lambda: c.attend(0, q, out, skip=-1),
           lambda: c.attend(0, rows((5, 3, 4, 64), 1), rows((5, 3, 4, 64), 1)),
           lambda: c.attend(0, rows((4, 3, 4, 68), 1)[..., 4:], out)]
    for call in bad:
        with pytest.raises(msf.MsfError) as e:
            call()
        assert e.value.status == msf.MSF_ERR_INVALID_ARG
    wrong = [lambda: c.attend(0, q[..., :32], out), lambda: c.attend(0, q.float(), out), lambda: c.attend(0, q, out[:3]),
             lambda: c.attend(0, q, out, lse.double()), lambda: c.attend(0, q, out, lse[:, :3]),
             lambda: c.attend(0, q, out, lse, seqs=ints([0, 1])),
             lambda: c.attend(0, q, out, lse, q.transpose(1, 2).contiguous().transpose(1, 2), lse)]
    for call in wrong:
        with pytest.raises(ValueError):
            call()
    ok(c)
    c.attend(0, q, out, lse, seqs=ints([0, 1, 4, -1]))  # a sequence that is none: said on the device, the row is empty
    ok(c, msf.MSF_ERR_INVALID_ARG)
    assert not out.any() and torch.isneginf(lse).all()
    c.attend(0, q[:, :0], out[:, :0])
    ok(c)
