"""Strides of dimensions of one may be anything, for every argument of the 4-bit cache's calls."""
import pytest
import torch

from cache_helpers import ints, make, ok, rows
from paper_2607_20940_gb300 import msf

pytestmark = pytest.mark.gpu


def one(x, dim, stride):
    """x with another stride in a dimension of one."""
    assert x.shape[dim] == 1
    st = list(x.stride())
    st[dim] = stride
    return x.as_strided(x.shape, st)


@pytest.mark.parametrize("dim,shape", [(0, (1, 5, 2, 64)), (1, (4, 1, 2, 64)), (2, (4, 5, 1, 64))])
def test_dimensions_of_one(dim, shape):
    n, tokens, heads, D = shape
    made = [make(kv_heads=heads, head_dim=D, sequences=n) for _ in range(3)]
    k, v, q = rows(shape, 1), rows(shape, 2), rows(shape, 3)
    got = []
    for c, ks, vs in zip(made, (None, 7, 7), (None, None, 3)):
        c.grow(None, None, tokens)
        c.write(0, k if ks is None else one(k, dim, ks), v if vs is None else one(v, dim, vs))
        k0, v0 = torch.empty_like(k), torch.empty_like(v)
        c.read(0, one(k0, dim, 5), v0)
        out, lse = torch.empty_like(q), torch.empty(n, heads, tokens, device="cuda")
        c.attend(0, one(q, dim, 9), one(out, dim, 1), lse)
        ok(c)
        got.append((k0, v0, out, lse))
    for other in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(got[0], other))


def test_refusals():
    c = make(kv_heads=2, head_dim=64, sequences=4)
    k, v = rows((4, 3, 2, 64), 1), rows((4, 3, 2, 64), 2)
    c.grow(None, None, 3)
    wide = rows((4, 6, 2, 64), 2)[:, ::2]
    with pytest.raises(ValueError, match="same strides"):
        c.write(0, k, wide)
    with pytest.raises(ValueError, match="shape"):
        c.write(0, k, rows((4, 4, 2, 64), 2))
    with pytest.raises(ValueError, match="bfloat16"):
        c.write(0, k, v.half())
    with pytest.raises(ValueError, match="device"):
        c.write(0, k, v.cpu())
    with pytest.raises(ValueError, match="contiguous"):
        c.write(0, rows((4, 3, 2, 128), 1)[..., ::2], rows((4, 3, 2, 128), 1)[..., ::2])
    with pytest.raises(msf.MsfError):
        c.write(0, rows((4, 3, 2, 68), 1)[..., :64], rows((4, 3, 2, 68), 1)[..., :64])
    with pytest.raises(ValueError, match="entries"):
        c.write(0, k, v, ints([0, 1]))
    ok(c)


def test_either_binding(monkeypatch):
    """The calls whose tensors are read in C and those that Python reads do the same and refuse the same."""
    assert msf._calls is not None, "built where Python's headers are"
    k, v, q = rows((3, 20, 2, 64), 1), rows((3, 20, 2, 64), 2), rows((3, 4, 6, 64), 3)
    base, base_lse = rows(q.shape, 4), torch.randn(3, 6, 4, device="cuda")
    got = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(msf, "_calls", None)
        c = make(kv_heads=2, head_dim=64, sequences=3)
        c.grow(None, ints([20, 3, 7]))
        c.write(0, k, v, ints([0, 1, 2]), ints([20, 3, 7]))
        k0, v0 = torch.empty_like(k), torch.empty_like(v)
        c.read(0, k0, v0, ints([2, 0, 1]), ints([1, 0, 2]))
        out, lse, joined, inside = torch.empty_like(q), torch.empty_like(base_lse), base.clone(), base_lse.clone()
        c.attend(0, q, out, lse, seqs=ints([2, 2, 0]), causal=True, softmax_scale=0.3, skip=1)
        c.attend(0, q, joined, inside, joined, inside, causal=False)
        other = torch.empty_like(q)
        c.attend(0, q, other, None, base, base_lse, simt=True)
        ok(c)
        got.append((k0, v0, out, lse, joined, inside, other))
        for refused in (lambda: c.write(1, k, v), lambda: c.write(0, k, v, None, None, stream=0) or c.read(-1, k0, v0),
                        lambda: c.attend(0, q, out, lse, skip=-1), lambda: c.attend(0, q, out, lse, base)):
            with pytest.raises(msf.MsfError):
                refused()
        for refused in (lambda: c.attend(0, q[0], out, lse), lambda: c.attend(0, q, out[:, :3], lse),
                        lambda: c.attend(0, q, out, lse.half()), lambda: c.attend(0, q, out, lse, base[:2], base_lse),
                        lambda: c.attend(0, q, out, lse, seqs=ints([0])), lambda: c.read(0, k0[..., :32], v0[..., :32])):
            with pytest.raises(ValueError):
                refused()
    assert all(torch.equal(x, y) for x, y in zip(*got))
