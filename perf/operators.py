"""Performance cases of the 4-bit key/value cache: what a program does with it.

The cache holds the keys and values of many sequences (streams, scales of a stream, beams)
in pages, each value as a 4-bit floating point number (one sign, two exponent and one
mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) with an 8-bit scale (e4m3) for every 16 values
along the head. The operators:

  append   quantises new tokens into their sequences' pages, and reads them back as values
  attend   attention of queries over the sequences' tokens, alone or joined with a partial
           attention over other keys (the window's, the sink's) by its log-sum-exp
  fork     sequences continue other sequences' pages (beams, streams that branch), and grow
           by a token each, which copies shared last pages
  copy     sequences become copies of others, with pages of their own
  compact  pages in use move down to the lowest numbers

The last three move pages whole and never look into them: their cases fill the pool with any
bytes and compare it byte for byte.

Sizes are the repository's workloads (the 480p layer: frames of 30 x 52 tokens, 12 heads x
128) and generic ones of language models: grouped heads, single tokens, prompts, ragged and
empty sequences.
"""
import math
import random

import torch

own = False

BLOCK = 16  # values that share a scale


def _attend(name, seqs, kv, group, dim, queries, longest, page, causal=0, base=0, ragged=1):
    c = {"op": "attend", "seqs": seqs, "kv": kv, "group": group, "dim": dim, "queries": queries, "longest": longest,
         "page": page, "causal": causal, "base": base, "ragged": ragged}
    return c if name is None else dict(c, name=name)


def _append(name, seqs, kv, dim, tokens, before, page, exp=0, ragged=1):
    c = {"op": "append", "seqs": seqs, "kv": kv, "dim": dim, "tokens": tokens, "before": before, "page": page,
         "exp": exp, "ragged": ragged}
    return c if name is None else dict(c, name=name)


def _pages(name, op, seqs, kv, dim, longest, page, layers, beams=1):
    c = {"op": op, "seqs": seqs, "kv": kv, "dim": dim, "longest": longest, "page": page, "layers": layers,
         "beams": beams}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # Two short streams, one of them still empty: latency is all there is.
        _attend("attend_tiny", 2, 2, 1, 64, 1, 60, 16),
        # Single tokens of a served batch: grouped heads, sequences of any age.
        _attend("decode_64x8k", 64, 8, 4, 128, 1, 8191, 32),
        # One user's token over a very long context: few rows, the work is split along it.
        _attend("decode_1x131k", 1, 8, 8, 128, 1, 131071, 64, ragged=0),
        # A few drafted tokens a sequence, checked together.
        _attend("verify_16x5", 16, 4, 4, 64, 5, 8000, 16, causal=1),
        # The next piece of prompts whose beginning is cached; the shortest is shorter than the piece.
        _attend("prompt_3x1000", 3, 4, 4, 128, 1000, 5099, 32, causal=1),
        # The fine states of the 480p window over sixteen frames of history, joined with the
        # attention over the window itself.
        _attend("window_480p", 1, 12, 1, 128, 3120, 24960, 64, base=1, ragged=0),
        # A token of every sequence of a served batch.
        _append("append_64x1", 64, 8, 128, 1, 3000, 32),
        # The head state that a step of the 480p window emits.
        _append("append_480p", 1, 12, 128, 1560, 23400, 64, ragged=0),
        # Prompts of a batch.
        _append("append_8x4096", 8, 8, 128, 4096, 77, 32),
        # A step of beam search: beams go on from others, then every one gets room for a token.
        _pages("fork_128", "fork", 128, 8, 128, 4001, 32, 4, beams=8),
        # Three streams of the 480p layer with eight frames of history branch for good.
        _pages("copy_480p", "copy", 3, 12, 128, 12480, 64, 2),
        # Half of the sequences have ended; what is left moves together.
        _pages("compact_256", "compact", 256, 8, 128, 4000, 16, 2),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case: the same operators over the whole range of sizes, odd ones included."""
    most = {op: max((work(c) for c in listed() if c["op"] == op), key=lambda w: w["bytes"]) for op in
            ("append", "fork", "copy", "compact")}
    while True:
        op = rng.choice(["attend"] * 6 + ["append"] * 3 + ["fork", "copy", "compact"])
        dim, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
        kv = rng.choice([1, 2, 4, 8, 12, rng.randint(1, 16)])
        if op == "attend":
            queries = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 2, 4000), _log(rng, 2, 4000)])
            c = _attend(None, _log(rng, 1, 128), kv, rng.choice([1, 1, 2, 3, 4, 5, 8, 16]), dim, queries,
                        _log(rng, 1, 200000), page, causal=rng.randint(0, 1), base=rng.randint(0, 1),
                        ragged=rng.choice([0, 1, 1]))
            w = work(c)
            rows = c["seqs"] * kv * c["longest"]
            if w["flops"] <= 478e9 and w["bytes"] <= 4e8 and rows * dim <= 4e8 and rows * c["group"] * queries <= 9e8:
                return c
            continue
        if op == "append":
            c = _append(None, _log(rng, 1, 128), kv, dim, _log(rng, 1, 5000), rng.choice([0, _log(rng, 1, 5000)]), page,
                        exp=rng.choice([0, 0, rng.randint(-6, 6)]), ragged=rng.choice([0, 1, 1]))
            if c["seqs"] * (c["tokens"] + c["before"]) * kv * dim > 1e8:
                continue
        else:
            beams = rng.choice([2, 3, 4, 5, 8]) if op == "fork" else 1
            c = _pages(None, op, beams * _log(rng, 1, 16 if op == "fork" else 24 if op == "copy" else 300), kv, dim,
                       _log(rng, 2, 20000), page, rng.randint(1, 4), beams)
            if _pool_pages(c) * c["layers"] * _page_bytes(c) > 1.3e9:
                continue
        if work(c)["bytes"] <= most[op]["bytes"]:
            return c


# ---------------------------------------------------------------- shapes

def _lengths(c):
    """Tokens of every sequence. Ragged: from none to the longest; an age is a matter of the case, not of the seed."""
    n, top = c["seqs"], c["longest"]
    if c["op"] == "attend" and not c["ragged"]:
        return [top] * n
    r = random.Random(n * 1000003 + top)
    got = [r.randint(1, top) for _ in range(n)]
    got[0] = top
    if c["op"] == "attend" and n > 1:
        got[1] = 0  # a sequence that has not begun
    if c["op"] == "attend" and n > 2:
        got[2] = min(top, max(1, c["queries"] // 2))
    return got


def _counts(c):
    """New tokens of every sequence, and the tokens before them."""
    n, t, b = c["seqs"], c["tokens"], c["before"]
    if not c["ragged"]:
        return [t] * n, [b] * n
    r = random.Random(n * 1000003 + t)
    return [t] + [r.randint(0 if t > 1 else 1, t) for _ in range(n - 1)], [r.randint(0, b) for _ in range(n)]


def _page_bytes(c):
    return c["kv"] * c["page"] * c["dim"] * 9 // 8  # a byte and an eighth for a key's and a value's 4 bits and scales


def _parts(c):
    """fork: the parent of each beam; compact: the sequences that have ended."""
    r = random.Random(c["seqs"] * 7919 + c["longest"])
    if c["op"] == "fork":
        k = c["beams"]
        return [i // k * k + r.randrange(k) for i in range(c["seqs"])]
    return sorted(r.sample(range(c["seqs"]), c["seqs"] // 2))


def _need(length, page):
    return -(-length // page)


def _pool_pages(c):
    """Pages of the pool that a program sets up for the case."""
    pages = sum(_need(x, c["page"]) for x in _lengths(c))
    if c["op"] == "fork":  # prompts, a page of its own for every beam before, and for every one after
        return sum(_need(x, c["page"]) for x in _lengths(c)[::c["beams"]]) + 4 * c["seqs"] + 8
    return 3 * pages + 8 if c["op"] == "copy" else pages + 8


def work(case):
    c = case
    D, Hk = c["dim"], c["kv"]
    token = 2 * Hk * D * 9 // 16  # a token's keys and values in the cache
    if c["op"] == "attend":
        H, nq = Hk * c["group"], c["queries"]
        keys = 0
        for n in _lengths(c):
            if c["causal"]:
                first = min(nq, max(0, nq - n))  # queries before the first key
                k = nq - first
                keys += k * n - k * (k - 1) // 2
            else:
                keys += nq * n
        bytes_ = sum(_lengths(c)) * token + c["seqs"] * nq * H * (4 * D + 4)
        if c["base"]:
            bytes_ += c["seqs"] * nq * H * (2 * D + 4)
        return {"bytes": bytes_, "flops": 4 * D * H * keys}
    if c["op"] == "append":
        n = sum(_counts(c)[0])
        return {"bytes": n * (4 * Hk * D + token) + n * token + c["seqs"] * c["tokens"] * 4 * Hk * D, "flops": 0}
    lens, P = _lengths(c), c["page"]
    data = c["layers"] * _page_bytes(c)
    if c["op"] == "fork":
        # tables read and written, and the shared last pages copied
        k = c["beams"]
        pages = [_need(lens[i // k * k], P) for i in range(c["seqs"])]
        copied = sum(1 for i in range(c["seqs"]) if lens[i // k * k] % P)
        return {"bytes": sum(pages) * 8 + 2 * copied * data, "flops": 0}
    if c["op"] == "copy":
        return {"bytes": sum(_need(x, P) for x in lens) * (8 + 2 * data), "flops": 0}
    ended, live, at, used = set(_parts(c)), 0, 0, []
    for i, x in enumerate(lens):
        n = _need(x, P)
        if i not in ended:
            used.append((at, at + n))
            live += n
        at += n
    moved = sum(max(0, z - max(a, live)) for a, z in used)
    return {"bytes": live * 8 + moved * 2 * data, "flops": 0}


# ----------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _tokens(c, gen, n, length):
    """Keys and values [n, length, heads, dim] as a model makes them: channels of the keys differ in size, and one in
    sixteen or so is several times the others."""
    Hk, D = c["kv"], c["dim"]
    gain = torch.exp2(_randn(gen, Hk, D) * 0.5) * torch.where(torch.rand(Hk, D, generator=gen, device="cuda") < 0.06, 3.0, 0.7)
    k = torch.empty(n, length, Hk, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    for i in range(n):
        k[i] = _randn(gen, length, Hk, D) * gain
        v[i] = _randn(gen, length, Hk, D)
    return k, v


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _inputs(c, seed):
    gen = _gen(seed)
    if c["op"] == "attend":
        H, nq, D = c["kv"] * c["group"], c["queries"], c["dim"]
        x = {}
        gain = torch.exp2(torch.rand(H, 1, generator=gen, device="cuda") * 2 - 1)
        x["q"] = (_randn(gen, c["seqs"], nq, H, D) * gain).to(torch.bfloat16)
        if c["base"]:
            x["base"] = (_randn(gen, c["seqs"], nq, H, D) * 0.1).to(torch.bfloat16)
            x["base_lse"] = math.log(max(1.0, c["longest"] / 4)) + 1 + _randn(gen, c["seqs"], H, nq)
            if nq > 1:
                x["base_lse"][:, :, -1] = -math.inf  # a row that sees nothing of the other keys
        x["k"], x["v"] = _tokens(c, gen, c["seqs"], c["longest"])
        return x
    if c["op"] == "append":
        k, v = _tokens(c, gen, c["seqs"], c["tokens"])
        return {"k": k * 2.0 ** c["exp"], "v": v * 2.0 ** c["exp"]}
    return {"pool": torch.randint(0, 256, (c["layers"], _pool_pages(c), _page_bytes(c)), generator=gen, device="cuda",
                                  dtype=torch.uint8)}


def prepare(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    s = {"c": c, **x}
    if c["op"] == "attend":
        s["scale"] = 1 / math.sqrt(c["dim"])
        s["lens"] = _ints(_lengths(c))
        (_own_filled if own else _plain_filled)(c, s, seed)
        del s["k"], s["v"]
    elif c["op"] == "append":
        counts, before = _counts(c)
        s["counts"], s["before"] = _ints(counts), _ints(before)
        s["after"] = s["counts"] + s["before"]
        if own:
            s["cache"] = _own_cache(c, sum(_need(a + b, c["page"]) for a, b in zip(counts, before)), max(a + b for a, b in zip(counts, before)))
            s["cache"].grow(None, s["before"])
            s["cache"].grow(None, s["counts"])
            s["k_back"], s["v_back"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        else:
            _plain_empty(c, s, sum(_need(a + b, c["page"]) for a, b in zip(counts, before)), max(a + b for a, b in zip(counts, before)), seed)
    else:
        (_own_pages if own else _plain_pages)(c, s)
    return s


# ------------------------------------------------- the framework's operators

def _own_cache(c, pages, longest, layers=1, seqs=None, pool=None):
    from paper_2607_20940_gb300 import msf
    cache = msf.Cache(msf.make_cache_desc(layers, c["kv"], c["dim"], c["page"], max(1, pages), seqs or c["seqs"],
                                          max(1, _need(longest, c["page"])), k_exponent=c.get("exp", 0),
                                          v_exponent=c.get("exp", 0)))
    cache.bind(cache.pool() if pool is None else pool, cache.state(), cache.workspace())
    return cache


def _own_filled(c, s, seed):
    """The sequences as a server fills them: all grow by turns, so that their pages lie among each other."""
    lens, top = _lengths(c), c["longest"]
    cache = s["cache"] = _own_cache(c, sum(_need(x, c["page"]) for x in lens), top)
    step = max(256, -(-top // 16))
    for at in range(0, top, step):
        n = min(step, top - at)
        counts = torch.clamp(s["lens"] - at, 0, n).to(torch.int32)
        cache.grow(None, counts)
        cache.write(0, s["k"][:, at:at + n], s["v"][:, at:at + n], None, counts)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(c["seqs"], c["kv"] * c["group"], c["queries"], device="cuda")


def _own_pages(c, s):
    n, P, lens = c["seqs"], c["page"], _lengths(c)
    op = c["op"]
    cache = s["cache"] = _own_cache(c, _pool_pages(c), max(lens) + 1, c["layers"], 2 * n if op == "copy" else n, s["pool"])
    if op == "fork":
        k = c["beams"]
        first = list(range(0, n, k))
        cache.grow(_ints(first), _ints([lens[i] for i in first]))
        rest = [i for i in range(n) if i % k]
        cache.fork(_ints([i // k * k for i in rest]), _ints(rest))
        s["src"], s["dst"], s["keep"] = _ints(_parts(c)), _ints(list(range(n))), _ints([lens[i // k * k] for i in range(n)])
    elif op == "copy":
        s["src"], s["dst"] = _ints(list(range(n))), _ints(list(range(n, 2 * n)))
        cache.grow(s["src"], _ints(lens))
    else:
        cache.grow(None, _ints(lens))
        cache.truncate(_ints(_parts(c)))
        s["saved"] = cache.bound_state.clone()


def _own_run(s):
    c, cache = s["c"], s["cache"]
    op = c["op"]
    if op == "attend":
        cache.attend(0, s["q"], s["out"], s["lse"], s.get("base"), s.get("base_lse"), causal=bool(c["causal"]))
        return {"out": s["out"], "lse": s["lse"]}
    if op == "append":
        cache.write(0, s["k"], s["v"], None, s["counts"])
        cache.read(0, s["k_back"], s["v_back"], None, s["before"])
        return {"k": s["k_back"], "v": s["v_back"]}
    if op == "fork":
        cache.fork(s["src"], s["dst"], s["keep"])
        cache.grow(None, None, 1)
    elif op == "copy":
        cache.fork(s["src"], s["dst"], copy=True)
    else:
        cache.bound_state.copy_(s["saved"])
        cache.compact()
    return {"pool": s["pool"], "table": cache.table, "lengths": cache.lengths, "refs": cache.refs}


# ------------------------------------------------------------ the plain forms

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _plain_quantise(x, exp):
    """Codes [.., D/2] (two a byte, the lower first) and scales [.., D/16] of x [.., D]."""
    unit = 2.0 ** exp
    b = x.float().unflatten(-1, (-1, BLOCK))
    s = (b.abs().amax(-1, keepdim=True) / (6 * unit)).clamp(max=448.0).to(torch.float8_e4m3fn).float().clamp(min=2.0 ** -9)
    y = b / (s * unit)
    a = y.abs()
    # to the nearest, ties to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code + 8 * (y < 0)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, s.squeeze(-1).to(torch.float8_e4m3fn)


def _plain_values(codes, scales, exp=0):
    grid = torch.tensor(_GRID + tuple(-g for g in _GRID), device="cuda")
    v = grid[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (v.unflatten(-1, (-1, BLOCK)) * (scales.float() * 2.0 ** exp).unsqueeze(-1)).flatten(-2)


def _plain_empty(c, s, pages, longest, seed):
    P, Hk, D = c["page"], c["kv"], c["dim"]
    pages, W = max(1, pages), max(1, _need(longest, P))
    gen = _gen(seed + 1)
    need = -(-s.get("lens", s.get("after")) // P)
    at = torch.cumsum(need, 0) - need
    col = torch.arange(W, device="cuda")
    perm = torch.randperm(pages, generator=gen, device="cuda")
    s["table"] = torch.where(col < need[:, None], perm[(at[:, None] + col).clamp(max=pages - 1)], 0)
    for n in "kv":
        s[n + "_codes"] = torch.zeros(pages * P, Hk, D // 2, dtype=torch.uint8, device="cuda")
        s[n + "_scales"] = torch.zeros(pages * P, Hk, D // BLOCK, dtype=torch.float8_e4m3fn, device="cuda")


def _plain_filled(c, s, seed):
    _plain_empty(c, s, sum(_need(x, c["page"]) for x in _lengths(c)), c["longest"], seed)
    for i, n in enumerate(_lengths(c)):
        t = torch.arange(n, device="cuda")
        slot = s["table"][i][t // c["page"]] * c["page"] + t % c["page"]
        for m in "kv":
            codes, scales = _plain_quantise(s[m][i, :n], 0)
            s[m + "_codes"][slot] = codes
            s[m + "_scales"].view(torch.uint8)[slot] = scales.view(torch.uint8)


def _plain_gather(s, n, P):
    """[seqs, heads, tokens, dim] of the sequences' pages."""
    codes = s[n + "_codes"].unflatten(0, (-1, P))[s["table"]].flatten(1, 2)
    scales = s[n + "_scales"].view(torch.uint8).unflatten(0, (-1, P))[s["table"]].flatten(1, 2).view(torch.float8_e4m3fn)
    return _plain_values(codes.transpose(1, 2), scales.transpose(1, 2))


def _plain_attend(s):
    c = s["c"]
    Hk, r, D, nq, n = c["kv"], c["group"], c["dim"], c["queries"], c["seqs"]
    k = _plain_gather(s, "k", c["page"])
    q = s["q"].float().view(n, nq, Hk, r, D).permute(0, 2, 3, 1, 4).reshape(n, Hk, r * nq, D)
    score = (q @ k.transpose(-1, -2)) * s["scale"]
    del k
    key = torch.arange(score.shape[-1], device="cuda")
    lens = s["lens"].view(n, 1, 1, 1)
    last = lens + torch.zeros(1, 1, r * nq, 1, device="cuda", dtype=torch.int32)
    if c["causal"]:
        last = last - nq + 1 + torch.arange(nq, device="cuda").repeat(r).view(1, 1, -1, 1)
    score.masked_fill_(key >= last, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = _plain_gather(s, "v", c["page"])
    out = (p @ v) / torch.where(total == 0, 1.0, total)
    lse = top + total.log()
    out = out.view(n, Hk, r, nq, D).permute(0, 3, 1, 2, 4).reshape(n, nq, Hk * r, D)
    lse = lse.view(n, Hk * r, nq)
    if c["base"]:
        top = torch.maximum(lse, s["base_lse"])
        top = torch.where(top == -math.inf, 0.0, top)
        a, b = (lse - top).exp(), (s["base_lse"] - top).exp()
        w = torch.where(a + b == 0, 1.0, a + b)
        out = out * (a / w).transpose(1, 2)[..., None] + s["base"].float() * (b / w).transpose(1, 2)[..., None]
        lse = top + (a + b).log()
    return {"out": out.to(torch.bfloat16), "lse": lse}


def _plain_append(s):
    c = s["c"]
    t = torch.arange(c["tokens"], device="cuda")
    here = t < s["counts"][:, None]
    pos = (s["before"][:, None] + t).long()
    slot = (torch.gather(s["table"], 1, (pos // c["page"]).clamp(max=s["table"].shape[1] - 1)) * c["page"] + pos % c["page"])[here]
    back = {}
    for n in "kv":
        codes, scales = _plain_quantise(s[n][here], c["exp"])
        s[n + "_codes"][slot] = codes
        s[n + "_scales"].view(torch.uint8)[slot] = scales.view(torch.uint8)
        got = torch.zeros_like(s[n])
        got[here] = _plain_values(s[n + "_codes"][slot], s[n + "_scales"].view(torch.uint8)[slot].view(torch.float8_e4m3fn), c["exp"]).to(torch.bfloat16)
        back[n] = got
    return back


def _plain_free(refs, n):
    return torch.nonzero(refs == 0).flatten()[:n]


def _plain_grow(s, seqs, counts):
    """Room for counts[i] more tokens of sequence seqs[i]: pages that are free, the lowest first; a shared last page that
    is not full is copied."""
    P, table, lens, refs = s["c"]["page"], s["table"], s["lens"], s["refs"]
    col = torch.arange(table.shape[1], device="cuda")
    old, new = lens[seqs], lens[seqs] + counts
    rows = table[seqs]
    tail = (old // P)[:, None]
    part = (old % P != 0) & (counts > 0)
    shared = part & (refs[torch.gather(rows, 1, tail.clamp(max=col.numel() - 1).long()).flatten().clamp(min=0)] > 1)
    take = (col >= -(-old // P)[:, None]) & (col < -(-new // P)[:, None]) | (col == tail) & shared[:, None]
    free = _plain_free(refs, int(take.sum())).to(torch.int32)
    src, dst = rows[(col == tail) & shared[:, None]].long(), None
    rows[take] = free
    dst = rows[(col == tail) & shared[:, None]].long()
    s["pool"][:, dst] = s["pool"][:, src]
    refs.index_add_(0, src, torch.full_like(src, -1, dtype=torch.int32))
    refs[free.long()] = 1
    table[seqs] = rows
    lens[seqs] = new


def _plain_fork(s, src, dst, keep, copy=False):
    P, table, lens, refs = s["c"]["page"], s["table"], s["lens"], s["refs"]
    col = torch.arange(table.shape[1], device="cuda")
    new = lens[src] if keep is None else torch.minimum(lens[src], keep)
    has = col < -(-new // P)[:, None]
    rows = torch.where(has, table[src], -1)
    if copy:
        free = _plain_free(refs, int(has.sum())).to(torch.int32)
        s["pool"][:, free.long()] = s["pool"][:, rows[has].long()]
        rows[has] = free
    old = table[dst]
    old = old[old >= 0].long()
    refs.index_add_(0, old, torch.full_like(old, -1, dtype=torch.int32))
    refs.index_add_(0, rows[has].long(), torch.ones_like(rows[has]))
    table[dst] = rows
    lens[dst] = new


def _plain_truncate(s, seqs):
    table, refs = s["table"], s["refs"]
    old = table[seqs]
    old = old[old >= 0].long()
    refs.index_add_(0, old, torch.full_like(old, -1, dtype=torch.int32))
    table[seqs] = -1
    s["lens"][seqs] = 0


def _plain_compact(s):
    refs, table = s["refs"], s["table"]
    live = int((refs > 0).sum())
    hole = torch.nonzero(refs[:live] == 0).flatten()
    high = torch.nonzero(refs[live:] > 0).flatten() + live
    to = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
    to[high] = hole.to(torch.int32)
    s["pool"][:, hole] = s["pool"][:, high]
    refs[hole] = refs[high]
    refs[high] = 0
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], table))


def _plain_pages(c, s):
    n, lens, op = c["seqs"], _lengths(c), c["op"]
    S = 2 * n if op == "copy" else n
    s["table"] = torch.full((S, _need(max(lens) + 1, c["page"])), -1, dtype=torch.int32, device="cuda")
    s["lens"] = torch.zeros(S, dtype=torch.int32, device="cuda")
    s["refs"] = torch.zeros(_pool_pages(c), dtype=torch.int32, device="cuda")
    if op == "fork":
        k = c["beams"]
        first = list(range(0, n, k))
        _plain_grow(s, _ints(first).long(), _ints([lens[i] for i in first]))
        rest = [i for i in range(n) if i % k]
        _plain_fork(s, _ints([i // k * k for i in rest]).long(), _ints(rest).long(), None)
        s["src"], s["dst"], s["keep"] = _ints(_parts(c)).long(), torch.arange(n, device="cuda"), _ints([lens[i // k * k] for i in range(n)])
    elif op == "copy":
        s["src"], s["dst"] = torch.arange(n, device="cuda"), torch.arange(n, 2 * n, device="cuda")
        _plain_grow(s, s["src"], _ints(lens))
    else:
        _plain_grow(s, torch.arange(n, device="cuda"), _ints(lens))
        _plain_truncate(s, _ints(_parts(c)).long())
        s["saved"] = [s[m].clone() for m in ("table", "lens", "refs")]


def _plain_run(s):
    op = s["c"]["op"]
    if op == "attend":
        return _plain_attend(s)
    if op == "append":
        return _plain_append(s)
    if op == "fork":
        _plain_fork(s, s["src"], s["dst"], s["keep"])
        _plain_grow(s, s["dst"], torch.ones_like(s["keep"]))
    elif op == "copy":
        _plain_fork(s, s["src"], s["dst"], None, copy=True)
    else:
        s["table"].copy_(s["saved"][0])
        s["lens"].copy_(s["saved"][1])
        s["refs"].copy_(s["saved"][2])
        _plain_compact(s)
    return {"pool": s["pool"], "table": s["table"], "lengths": s["lens"], "refs": s["refs"]}


def run(state):
    return _own_run(state) if own else _plain_run(state)


# --------------------------------------------------------------- in 64 bits

def _exact_quantised(x, exp):
    """What x [.., D] becomes in the cache, from the format's definition."""
    grid = torch.tensor(_GRID, dtype=torch.float64, device="cuda")
    b = x.double().unflatten(-1, (-1, BLOCK)) * 2.0 ** -exp
    want = b.abs().amax(-1, keepdim=True) / 6
    step = torch.exp2(torch.floor(torch.log2(want.clamp(min=2.0 ** -6, max=448.0))) - 3)  # e4m3's spacing there
    scale = (torch.round(want / step) * step).clamp(min=2.0 ** -9, max=448.0)
    a = (b.abs() / scale).clamp(max=6.0)
    up = torch.searchsorted(grid, a.contiguous()).clamp(max=7)
    down = (up - 1).clamp(min=0)
    over, under = grid[up] - a, a - grid[down]
    pick = torch.where((over < under) | (over == under) & (up % 2 == 0), up, down)
    return (torch.sign(b) * grid[pick] * scale).flatten(-2) * 2.0 ** exp


def exact(case, seed):
    c = dict(case)
    if c["op"] not in ("attend", "append"):
        return None  # page numbers and bytes: compared as they are
    x = _inputs(c, seed)
    if c["op"] == "append":
        t = torch.arange(c["tokens"], device="cuda")
        here = (t < _ints(_counts(c)[0])[:, None])[..., None, None]
        return {n: torch.stack([_exact_quantised(y, c["exp"]) for y in x[n]]) * here for n in "kv"}
    n, Hk, r, D, nq = c["seqs"], c["kv"], c["group"], c["dim"], c["queries"]
    out = torch.zeros(n, nq, Hk * r, D, dtype=torch.float64, device="cuda")
    lse = torch.full((n, Hk * r, nq), -math.inf, dtype=torch.float64, device="cuda")
    for i, length in enumerate(_lengths(c)):
        seen = torch.full((nq,), length, device="cuda")
        if c["causal"]:
            seen = (length - nq + 1 + torch.arange(nq, device="cuda")).clamp(min=0)
        hide = torch.arange(length, device="cuda")[None] >= seen[:, None]
        for g in range(Hk if length else 0):
            k, v = _exact_quantised(x["k"][i, :length, g], 0), _exact_quantised(x["v"][i, :length, g], 0)
            for h in range(g * r, g * r + r):
                z = (x["q"][i, :, h].double() @ k.T / math.sqrt(D)).masked_fill(hide, -math.inf)
                lse[i, h] = torch.logsumexp(z, 1)
                out[i, :, h] = torch.softmax(z, 1).nan_to_num(0.0) @ v
    if c["base"]:
        other = x["base_lse"].double()
        both = torch.logaddexp(lse, other)
        share = lambda l: torch.where(both == -math.inf, 0.0, torch.exp(l - both)).nan_to_num(0.0).transpose(1, 2)[..., None]  # noqa: E731
        out = out * share(lse) + x["base"].double() * share(other)
        lse = both
    return {"out": out, "lse": lse}
