"""Appending to the 4-bit cache and reading back, against the format in 64 bits: every
value held is exact in bf16, so what is read equals the oracle's bit for bit."""
import numpy as np
import pytest
import torch

from cache_helpers import f64, ints, make, ok, rows
from oracle import cache as oc
from paper_2607_20940_gb300 import msf

pytestmark = pytest.mark.gpu


def _held(x, exponent=0):
    return oc.quantise(f64(x), exponent)[0]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("steps", [(1,), (1, 1, 1), (15, 2), (16,), (37, 1, 90), (130,)])
def test_tokens_come_back(D, P, steps):
    c = make(layers=2, kv_heads=3, head_dim=D, page_tokens=P, sequences=2, sequence_pages=-(-160 // P), pages=40)
    ks, vs = [], []
    for i, n in enumerate(steps):
        k, v = rows((2, n, 3, D), 10 * i + 1, 2.0), rows((2, n, 3, D), 10 * i + 2, 0.3)
        c.grow(tokens=n)
        c.write(1, k, v)
        ks.append(k)
        vs.append(v)
    k, v = torch.cat(ks, 1), torch.cat(vs, 1)
    kb, vb = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    c.read(1, kb, vb)
    ok(c)
    assert np.array_equal(f64(kb), _held(k)) and np.array_equal(f64(vb), _held(v))
    # from the middle, past the end: zeros there
    kb, vb = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    at = sum(steps) // 2
    c.read(1, kb, vb, None, ints([at, -1]))
    n = sum(steps) - at
    assert np.array_equal(f64(kb)[0, :n], _held(k)[0, at:]) and not f64(kb)[0, n:].any()
    assert not f64(vb)[1, 0].any() and np.array_equal(f64(vb)[1, 1:], _held(v)[1, :-1])
    ok(c)


def test_ragged_counts_lists_and_strides():
    D, H, T = 128, 2, 40
    c = make(kv_heads=H, head_dim=D, sequences=5, sequence_pages=8, pages=40)
    first = [3, 0, 17, 30, 1]
    c.grow(None, ints(first))
    k0 = rows((5, 30, H, D), 1)
    c.write(0, k0, k0, None, ints(first))
    seqs, counts = [4, 0, 2], [40, 0, 15]
    big = rows((3, H, T + 2, 2 * D), 2)  # heads outside of tokens, every second head-sized run
    k = big[:, :, 1:T + 1, :D].transpose(1, 2)
    v = big[:, :, 1:T + 1, D:].transpose(1, 2)
    assert k.stride() == v.stride() and not k.is_contiguous()
    c.grow(ints(seqs), ints(counts))
    c.write(0, k, v, ints(seqs), ints(counts))
    kb = torch.empty(5, 60, H, D, dtype=torch.bfloat16, device="cuda")
    vb = torch.empty_like(kb)
    c.read(0, kb, vb)
    ok(c)
    want_k, want_v = np.zeros(kb.shape), np.zeros(kb.shape)
    for s, n in enumerate(first):
        want_k[s, :n] = want_v[s, :n] = _held(k0)[s, :n]
    for i, (s, n) in enumerate(zip(seqs, counts)):
        want_k[s, first[s]:first[s] + n] = _held(k)[i, :n]
        want_v[s, first[s]:first[s] + n] = _held(v)[i, :n]
    assert np.array_equal(f64(kb), want_k) and np.array_equal(f64(vb), want_v)


@pytest.mark.parametrize("exponent", [-64, -7, 0, 5, 64])
def test_sizes_of_values(exponent):
    """Ties of codes and scales, blocks of zeros, values below the smallest and above the largest scale."""
    D = 64
    c = make(head_dim=D, kv_heads=1, sequences=1, sequence_pages=40, pages=40, k_exponent=exponent, v_exponent=exponent)
    rng = np.random.default_rng(3)
    n = 600
    scale = rng.choice(oc.E4M3[1:], (n, 4, 1))
    mid = np.concatenate([oc.GRID, [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]])
    x = rng.choice(mid, (n, 4, 16)) * scale * rng.choice([-1, 1], (n, 4, 16))
    x[:100] = rng.standard_normal((100, 4, 16)) * np.exp2(rng.integers(-14, 12, (100, 4, 1)))
    x[100:110] = 0
    with np.errstate(over="ignore"):
        x = torch.from_numpy(x.reshape(1, n, 1, D) * 2.0 ** exponent).to(torch.float32).to(torch.bfloat16).cuda()
    c.grow(tokens=n)
    c.write(0, x, -x)
    kb, vb = torch.empty_like(x), torch.empty_like(x)
    c.read(0, kb, vb)
    ok(c)
    assert np.array_equal(f64(kb), _held(x, exponent)) and np.array_equal(f64(vb), -_held(x, exponent))


def test_values_that_are_not_finite():
    c = make(sequences=1, sequence_pages=4, pages=4)
    x = rows((1, 20, 2, 64), 1)
    x[0, 3, 1, 5], x[0, 3, 1, 30], x[0, 9, 0, 63], x[0, 9, 0, 62] = float("nan"), -float("inf"), float("inf"), float("nan")
    c.grow(tokens=20)
    c.write(0, x, x)
    kb, vb = torch.empty_like(x), torch.empty_like(x)
    c.read(0, kb, vb)
    ok(c, msf.MSF_ERR_NONFINITE)
    ok(c)
    assert np.array_equal(f64(kb), _held(x)) and np.array_equal(f64(vb), _held(x))
    assert np.isfinite(f64(kb)).all()


def test_shared_pages_are_not_written():
    c = make(sequences=2, sequence_pages=4, pages=8)
    x = rows((1, 20, 2, 64), 1)
    c.grow(ints([0]), None, 20)
    c.write(0, x, x, ints([0]))
    c.fork(ints([0]), ints([1]))
    y = rows((1, 20, 2, 64), 2)
    c.write(0, y, y, ints([1]))  # over pages that sequence 0 reads too
    ok(c, msf.MSF_ERR_INVALID_ARG)
    kb, vb = torch.empty_like(x), torch.empty_like(x)
    c.read(0, kb, vb, ints([0]))
    assert np.array_equal(f64(kb), _held(x))


def test_bad_lists_change_nothing():
    c = make(sequences=3, sequence_pages=4, pages=8)
    x = rows((3, 20, 2, 64), 1)
    c.grow(tokens=20)
    c.write(0, x, x)
    pool = c.bound_pool.clone()
    for seqs, counts in (([0, 3, 1], None), ([0, -1, 1], None), (None, [1, 21, 1]), (None, [1, -1, 1])):
        c.write(0, -x, -x, ints(seqs), ints(counts))
        ok(c, msf.MSF_ERR_INVALID_ARG)
        kb = torch.empty_like(x)
        c.read(0, kb, torch.empty_like(x))
        ok(c)
        sel = [1] if counts else [2]  # the row that is wrong touched no one
        assert np.array_equal(f64(kb)[sel], _held(x)[sel])
        c.write(0, x, x)
        ok(c)
    assert torch.equal(pool, c.bound_pool)


def test_refusals():
    c = make()
    x = rows((4, 3, 2, 64), 1)
    for call in (lambda: c.write(1, x, x), lambda: c.write(-1, x, x), lambda: c.read(1, x, x)):
        with pytest.raises(msf.MsfError) as e:
            call()
        assert e.value.status == msf.MSF_ERR_INVALID_ARG
    many = rows((5, 3, 2, 64), 1)  # more rows than sequences
    odd = rows((4, 3, 2, 68), 1)[..., :64]  # strides that are no multiples of 8
    off = rows((4 * 3 * 2 * 64 + 4,), 1)[4:].view(4, 3, 2, 64)  # 8-byte aligned
    for y in (many, odd, off):
        with pytest.raises(msf.MsfError) as e:
            c.write(0, y, y)
        assert e.value.status == msf.MSF_ERR_INVALID_ARG
    for k, v, seqs, counts in ((x.float(), x, None, None), (x, x[:3], None, None), (x[..., :32], x[..., :32], None, None),
                               (x, x, ints([0, 1, 2]), None), (x, x, None, torch.ones(4, device="cuda")),
                               (x.cpu(), x.cpu(), None, None), (x.transpose(1, 2), x.transpose(1, 2), None, None)):
        with pytest.raises(ValueError):
            c.write(0, k, v, seqs, counts)
    ok(c)
