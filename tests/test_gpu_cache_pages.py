"""Tables, references and pages of the 4-bit cache against the page model; the pages' bytes
follow (each page starts as bytes of its own number)."""
import random

import numpy as np
import pytest
import torch

from cache_helpers import ints, make, ok, same_tables
from oracle import cache as oc
from paper_2607_20940_gb300 import msf

pytestmark = pytest.mark.gpu


def _numbered(c):
    """Every page's every 4 bytes say where they are: layer, page."""
    d, info = c.desc, c.info
    pool = c.bound_pool.view(torch.int32).view(d.layers, d.pages, -1)
    pool.copy_((torch.arange(d.layers, device="cuda")[:, None, None] * 100000 +
                torch.arange(d.pages, device="cuda")[None, :, None]).int().expand_as(pool))
    return pool


def _same(c, pool, model):
    same_tables(c, model)
    want = torch.tensor(model.data, device="cuda", dtype=torch.int32)
    for layer in range(c.desc.layers):
        assert torch.equal(pool[layer], (layer * 100000 + want)[:, None].expand_as(pool[layer]))


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("P,pages,S,W,layers", [(16, 50, 5, 9, 2), (64, 33, 7, 6, 1), (32, 1100, 40, 70, 3),
                                               (128, 40000, 300, 200, 1)])
def test_any_order_of_operations(seed, P, pages, S, W, layers):
    rng = random.Random(seed)
    c = make(layers=layers, kv_heads=1, head_dim=64, page_tokens=P, pages=pages, sequences=S, sequence_pages=W)
    pool, m = _numbered(c), oc.Pages(pages, S, P, W)
    full = 0
    for step in range(24):
        op = rng.choice(["grow", "grow", "grow", "fork", "copy", "truncate", "compact"])
        some = rng.sample(range(S), rng.randint(1, S))
        top = W * P // 3
        want = msf.MSF_OK
        try:
            if op == "grow":
                counts = [rng.choice([0, 1, rng.randint(0, top)]) for _ in some]
                c.grow(ints(some), ints(counts))
                m.grow(some, counts)
            elif op in ("fork", "copy"):
                src = [rng.randrange(S) for _ in some]
                keep = rng.choice([None, [rng.randint(0, W * P) for _ in some]])
                c.fork(ints(src), ints(some), ints(keep), copy=op == "copy")
                m.fork(src, some, keep, op == "copy")
            elif op == "truncate":
                some = some[:max(1, len(some) // 2)]
                keep = rng.choice([None, [rng.randint(0, W * P) for _ in some]])
                c.truncate(ints(some), ints(keep))
                m.truncate(some, keep)
            else:
                c.compact()
                m.compact()
        except oc.Full:
            want, full = msf.MSF_ERR_PAGES, full + 1
        ok(c, want)
        _same(c, pool, m)


def test_a_list_may_permute():
    c = make(sequences=4, pages=30, sequence_pages=8)
    pool, m = _numbered(c), oc.Pages(30, 4, 16, 8)
    for s, n in enumerate((5, 40, 0, 100)):
        c.grow(ints([s]), None, n)
        m.grow([s], [n])
    for copy in (False, True):
        c.fork(ints([1, 2, 3, 0]), ints([0, 1, 2, 3]), copy=copy)
        m.fork([1, 2, 3, 0], [0, 1, 2, 3], None, copy)
        ok(c)
        _same(c, pool, m)


@pytest.mark.parametrize("what", ["grow", "fork", "truncate"])
@pytest.mark.parametrize("rows", [[0, 4], [0, -1], [1, 2, 1], [3, 3]])
def test_lists_that_are_wrong_change_nothing(what, rows):
    c = make(sequences=4, pages=30, sequence_pages=8)
    pool, m = _numbered(c), oc.Pages(30, 4, 16, 8)
    c.grow(None, ints([5, 40, 0, 100]))
    m.grow(range(4), [5, 40, 0, 100])

    def call(seqs, n):
        if what == "grow":
            c.grow(ints(seqs), ints(n))
        elif what == "fork":
            c.fork(ints([0] * len(seqs)), ints(seqs), ints(n))
        else:
            c.truncate(ints(seqs), ints(n))

    call(rows, [1] * len(rows))
    c.compact()  # and nothing follows until the status is read
    c.truncate()
    ok(c, msf.MSF_ERR_INVALID_ARG)
    _same(c, pool, m)
    call([0, 1], [1, -1])
    ok(c, msf.MSF_ERR_INVALID_ARG)
    if what == "fork":
        c.fork(ints([0, 9]), ints([1, 2]))
        ok(c, msf.MSF_ERR_INVALID_ARG)
    _same(c, pool, m)
    c.truncate()
    ok(c)
    assert not c.refs.any() and not c.lengths.any() and (c.table == -1).all()


def test_full_pool_and_full_table():
    c = make(sequences=3, pages=10, sequence_pages=8)
    c.grow(None, ints([128, 32, 0]))
    ok(c)
    before = c.bound_state.clone()
    c.grow(ints([2]), None, 1)  # no page left
    ok(c, msf.MSF_ERR_PAGES)
    c.grow(ints([0]), None, 1)  # no table entry left
    ok(c, msf.MSF_ERR_PAGES)
    c.grow(ints([0]), None, 0x7fffffff)
    ok(c, msf.MSF_ERR_PAGES)
    c.fork(ints([1]), ints([2]), copy=True)
    ok(c, msf.MSF_ERR_PAGES)
    assert torch.equal(before, c.bound_state)
    c.fork(ints([1]), ints([2]))
    ok(c)
    assert c.refs.tolist() == [1] * 8 + [2, 2]


def test_a_saved_state_goes_on():
    c = make(layers=2, sequences=3, pages=20, sequence_pages=8)
    pool, m = _numbered(c), oc.Pages(20, 3, 16, 8)
    c.grow(None, ints([50, 3, 90]))
    m.grow(range(3), [50, 3, 90])
    c.truncate(ints([0]))
    m.truncate([0])
    state, data = c.bound_state.clone(), c.bound_pool.clone()
    other = msf.Cache(c.desc)
    other.bind(other.pool(), other.state(), other.workspace())
    other.bound_pool.copy_(data)
    other.bound_state.copy_(state)
    for x in (c, other):
        x.compact()
        x.grow(ints([0]), None, 17)
        ok(x)
    m.compact()
    m.grow([0], [17])
    _same(c, pool, m)
    assert torch.equal(c.bound_state, other.bound_state) and torch.equal(c.bound_pool, other.bound_pool)


def test_graph_replays():
    """A captured step (fork, grow, compact) goes on from whatever the tables hold."""
    c = make(layers=2, sequences=4, pages=60, sequence_pages=12)
    pool, m = _numbered(c), oc.Pages(60, 4, 16, 12)
    c.grow(None, ints([5, 40, 0, 100]))
    m.grow(range(4), [5, 40, 0, 100])
    src, dst, keep = ints([3, 3]), ints([0, 2]), ints([30, 200])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.fork(src, dst, keep)
        c.grow(None, None, 7)
        c.compact()
    for _ in range(4):
        g.replay()
        m.fork([3, 3], [0, 2], [30, 200])
        m.grow(range(4), [7] * 4)
        m.compact()
        ok(c)
        _same(c, pool, m)


def test_refusals():
    c = make()
    for call in (lambda: c.grow(tokens=-1), lambda: c.grow(ints(range(5)), None, 1),
                 lambda: msf.msf_cache_fork(c.handle, ints([0]), ints([1]), None, 2)):
        with pytest.raises(msf.MsfError) as e:
            call()
        assert e.value.status == msf.MSF_ERR_INVALID_ARG
    for call in (lambda: c.fork(ints([0]), ints([1, 2])), lambda: c.truncate(ints([0]), ints([1, 2])),
                 lambda: c.grow(torch.zeros(2, device="cuda")), lambda: c.grow(torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()
    c.grow(ints([]), None, 3)
    c.truncate(ints([]))
    ok(c)
