"""A rollout with its whole history in 4 bits, against Eq. 4's softmax in 64 bits over sink, the
history's values as the cache holds them (subsampled, then quantised) and the window.

Bounds: two bf16 roundings of the output (the window's part and the joined one), and of the
probabilities (2^-9 relative) and the subsampled window rows: the bf16 attention's bounds, max 2e-2
and mean 2e-3 for values of unit variance, as everywhere in these tests."""
import numpy as np
import pytest
import torch

from cache_helpers import f64, rows
from oracle import cache as oc
from oracle import mssa
from paper_2607_20940_gb300 import msf
from paper_2607_20940_gb300.long_history import LongHistory, main

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(x).to(torch.float32).to(torch.bfloat16).double().numpy()


def expected(scales, gh, gw, q, k, v, sink, past):
    """past: {scale: (keys, values)} [B, tokens, H, D] of the history, as held."""
    B, _, H, D = q.shape
    counts = [gh * gw // (s * s) for s in scales]
    at = np.cumsum([0] + counts)
    out = np.zeros(q.shape)
    for g in sorted(set(scales)):
        ctx = []
        for x, which in ((k, 0), (v, 1)):
            parts = [sink[which], past[g][which]]
            for i, s in enumerate(scales):
                state = x[:, at[i]:at[i + 1]]
                parts.append(mssa.resample(state, gh // s, gw // s, g // s) if s < g else state)
            ctx.append(np.concatenate(parts, 1))
        for i, s in enumerate(scales):
            if s == g:
                z = np.einsum("bqhd,bkhd->bhqk", q[:, at[i]:at[i + 1]], ctx[0]) / np.sqrt(D)
                p = np.exp(z - z.max(-1, keepdims=True))
                out[:, at[i]:at[i + 1]] = np.einsum("bhqk,bkhd->bqhd", p / p.sum(-1, keepdims=True), ctx[1])
    return out


@pytest.mark.parametrize("scales,gh,gw,D", [((1, 1, 2), 8, 8, 64), ((1, 2, 4), 8, 12, 128), ((1, 1), 6, 10, 64)])
def test_rollout_with_a_branch(scales, gh, gw, D):
    H, B, sink_n, layers = 2, 2, 20, 2
    h = LongHistory(scales, gh, gw, H, D, sink_n, layers, batch=B, streams=3, frames=20, stream_frames=8, page_tokens=16)
    sinks = []
    for layer in range(layers):
        s = [rows((B, sink_n, H, D), 100 + 2 * layer + i) for i in range(2)]
        h.bind_sink(layer, *s)
        sinks.append([f64(x) for x in s])
    n, G = h.info.n_tokens, gh * gw
    groups = sorted(set(scales))
    past = [{s: {g: [np.zeros((0, H, D))] * 2 for g in groups} for s in range(3)} for _ in range(layers)]
    out, lse = torch.empty(B, n, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, n, device="cuda")
    seed = 0
    for step, streams in enumerate([(0, 1), (0, 1), (2, 1), (0, 2), (1, 2)]):
        if step == 2:
            h.branch([0], [2])
            for layer in range(layers):
                past[layer][2] = dict(past[layer][0])
        if step == 4:
            h.rewind([1], [1])
            h.end([0])
            h.cache.compact()
            for layer in range(layers):
                past[layer][1] = {g: [x[:G // (g * g)] for x in past[layer][1][g]] for g in groups}
        w = h.window(streams)
        emitting = step != 3  # one pass that emits nothing
        if emitting:
            h.emit(w)
        for layer in range(layers):
            q, k, v = (rows((B, n, H, D), 1000 + 10 * seed + i) for i in range(3))
            seed += 1
            h.attend(layer, w, q, k, v, out, lse, emitting)
            held = {g: [np.stack([past[layer][s][g][i] for s in streams]) if len({len(past[layer][s][g][0]) for s in streams}) == 1
                        else [past[layer][s][g][i] for s in streams] for i in range(2)] for g in groups}
            for b in range(B):
                one = lambda x: x[b:b + 1]  # noqa: E731
                want = expected(scales, gh, gw, one(f64(q)), one(f64(k)), one(f64(v)), [one(x) for x in sinks[layer]],
                                {g: [np.asarray(held[g][i][b])[None] for i in range(2)] for g in groups})
                e = np.abs(one(f64(out)) - want)
                assert e.max() <= 2e-2 and e.mean() <= 2e-3, (step, layer, b, e.max(), e.mean())
            if emitting:
                h.append(layer, w, k, v)
                for b, s in enumerate(streams):
                    for g in groups:
                        new = [oc.quantise(bf16(mssa.resample(f64(x)[b:b + 1, :G], gh, gw, g)[0]))[0] for x in (k, v)]
                        past[layer][s][g] = [np.concatenate([a, y]) for a, y in zip(past[layer][s][g], new)]
    h.check()
    lengths = h.cache.lengths.tolist()
    for s in range(3):
        for i, g in enumerate(groups):
            assert lengths[s * len(groups) + i] == (0 if s == 0 else len(past[0][s][g][0]))


def test_example(capsys):
    main()
    assert "pages in use" in capsys.readouterr().out


def test_refusals():
    with pytest.raises(ValueError):
        LongHistory((2, 2), 8, 8, 2, 64, 0)
    h = LongHistory((1, 2), 8, 8, 2, 64, 0, batch=2, streams=2, frames=2, stream_frames=2)
    with pytest.raises(ValueError):
        h.window([0])
    h.bind_sink(0, None, None)
    w = h.window([0, 1])
    for _ in range(3):
        h.emit(w)
    with pytest.raises(msf.MsfError) as e:
        h.check()
    assert e.value.status == msf.MSF_ERR_PAGES
