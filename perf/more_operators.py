"""Timed cases of what a decoding or verification step over long contexts needs around the paged cache: page tables and slot maps from the lengths
that the sequences are to have, rotary positions on the way into the cache, and attention over the pages that a cheap score selects.

listed() are the fixed cases, draw() gives more of the same ranges.  prepare() makes a program's inputs; run() is one pass, in plain torch operations, or
through the library's entry points where `own` is true; exact() is what the outputs are in 64 bits.

A batch is described the way the entry points take it: rows start[s] .. start[s + 1] - 1 of the packed tensors are the last positions of sequence s,
length[s] is its length with them, pages[s] are the pages that hold it.
"""
import math

import torch

own = False

TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2.0, "fp16": 2.0, "int8": 1.0, "e4m3": 1.0}
QMAX = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100          # rows without an element that large are stored as zeros


def listed():
    return [
        # a verification round of a full batch: nine rows each, some sequences cross into a page or fall back out of one
        pages("pages_round", 1, 64, 16, 8000, "round"),
        # continuous batching: an eighth of the sequences end, as many prompts come in, the others go on by a token
        pages("pages_admit", 2, 1024, 64, 6000, "admit"),
        # one token of a small draft model: a single short call in a chain of them
        rotate("rotate_token", "rotate_write", 3, [1], [1500], 16, 2, 64, 64, 16, "bf16", "bf16"),
        # a decoding batch into an 8-bit cache, frequencies scaled by bands for a longer context
        rotate("rotate_decode", "rotate_write", 4, [1] * 64, _spread(64, 300, 2500), 32, 8, 128, 128, 64, "bf16", "e4m3", scaling="bands"),
        # prompts: 2880 image tokens and 128 words each, queries, keys and values as columns of one fused projection
        rotate("rotate_prompt", "rotate_write", 5, [3008] * 8, [3008] * 8, 32, 8, 128, 128, 64, "bf16", "bf16"),
        # image tokens that a selection has kept, at their own places in time, height and width; a quarter of each head has none; pairs next to each other
        rotate("rotate_image", "rotate", 6, [320] * 64, [320] * 64, 16, 16, 128, 96, 16, "fp16", "fp16", axes=3, interleaved=True),
        # the keys of whole prompts summarised, page by page
        sparse("summary_prompt", "summary", 7, [3008] * 8, [3008] * 8, 8, 8, 128, 64, "bf16", "bf16", 32),
        # one interactive sequence of a small model, one token
        sparse("sparse_token", "sparse", 8, [1], [32001], 16, 2, 64, 16, "bf16", "bf16", 64),
        # a decoding batch behind long contexts, 8-bit cache
        sparse("sparse_decode", "sparse", 9, [1] * 64, _spread(64, 9000, 61000), 32, 8, 128, 64, "bf16", "e4m3", 32),
        # drafted trees of eight tokens under verification
        sparse("sparse_tree", "sparse", 10, [8] * 16, _spread(16, 12000, 48000), 64, 8, 128, 32, "bf16", "bf16", 48, tree=True),
        # four drafted tokens behind a million
        sparse("sparse_long", "sparse", 11, [4], [1000003], 32, 4, 128, 64, "fp16", "int8", 128),
        # sequences short and long together, every head with keys of its own
        sparse("sparse_mixed", "sparse", 12, [1, 3, 1, 5, 0, 2], [4001, 77, 23001, 9001, 50, 2], 32, 32, 96, 128, "fp16", "e4m3", 8),
    ]


def _spread(n, lo, hi):
    """n lengths between lo and hi, in no order."""
    return [lo + (i * 7919 + 13) % n * (hi - lo) // max(n - 1, 1) for i in range(n)]


def _text(values):
    return ",".join(str(v) for v in values)


def _list(text):
    return [int(v) for v in text.split(",")]


def _named(name, c):
    return dict(c, name=name) if name else c


def pages(name, id, S, page, most, change, tight=False):
    return _named(name, dict(kind="pages", id=id, S=S, page=page, most=most, change=change, tight=tight))


def rotate(name, kind, id, new, length, heads, kv_heads, D, R, page, dtype, kept, axes=1, interleaved=False, scaling="plain"):
    return _named(name, dict(kind=kind, id=id, new=_text(new), length=_text(length), heads=heads, kv_heads=kv_heads, D=D, R=R, page=page, dtype=dtype, kept=kept,
                             axes=axes, interleaved=interleaved, scaling=scaling))


def sparse(name, kind, id, new, length, heads, kv_heads, D, page, dtype, kept, top, tree=False):
    return _named(name, dict(kind=kind, id=id, new=_text(new), length=_text(length), heads=heads, kv_heads=kv_heads, D=D, page=page, dtype=dtype, kept=kept, top=top,
                             first=1, recent=2 if page >= 64 else 4, tree=tree))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    u, id = rng.random(), rng.randint(100, 1 << 20)
    if u < 0.2:
        S = _log(rng, 1, 1024)
        return pages(None, id, S, rng.choice([16, 32, 64, 128]), _log(rng, 100, 6000), rng.choice(["round", "admit"]), rng.random() < 0.3)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    D, page = rng.choice([64, 96, 128, 128]), rng.choice([16, 32, 64, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    heads = kv_heads * rng.choice([1, 2, 4, 5, 8])
    if u < 0.55:
        S = _log(rng, 1, 64)
        new = [_log(rng, 1, max(1, 16000 // S)) for _ in range(S)] if rng.random() < 0.5 else [rng.choice([0, 1, 1, 1, rng.randint(2, 9)]) for _ in range(S - 1)] + [1]
        length = [n + rng.choice([0, rng.randint(0, 2000)]) for n in new]
        R = 16 * rng.randint(1, D // 16) if rng.random() < 0.3 else D
        kind = rng.choice(["rotate", "rotate_write", "rotate_write"])
        return rotate(None, kind, id, new, length, heads, min(kv_heads, heads), D, R, page, dtype, rng.choice([dtype, "e4m3"]), rng.choice([1, 1, 2, 3, 4]),
                      rng.random() < 0.4, rng.choice(["plain", "linear", "base", "bands", "ramp"]))
    if u < 0.65:
        S = _log(rng, 1, 32)
        new = [_log(rng, 1, max(1, 20000 // S)) for _ in range(S)]
        length = [n + rng.choice([0, rng.randint(0, 2000)]) for n in new]
        kv_heads = min(kv_heads, 8)
        return sparse(None, "summary", id, new, length, kv_heads, kv_heads, D, page, dtype, rng.choice([dtype, "int8", "e4m3"]), 16)
    S = _log(rng, 1, 64)
    n = 1 if rng.random() < 0.5 else rng.randint(2, 8)
    tree = n > 1 and rng.random() < 0.4
    new = [n if tree or rng.random() < 0.8 else rng.randint(0, n) for _ in range(S - 1)] + [n]
    # as many rows of scores and positions, and as large a cache, as the listed ones
    most = min(120000, 20000000 // (S * kv_heads), page * 1500000 // (sum(new) * kv_heads))
    length = [m + _log(rng, 100, max(200, most)) for m in new]
    top = max(8, min(rng.choice([8, 16, 32, 64, 100]), 1500000 // (sum(new) * kv_heads * page)))
    return sparse(None, "sparse", id, new, length, heads, kv_heads, D, page, dtype, rng.choice([dtype, "int8", "e4m3"]), top, tree)


# ---------------------------------------------------------------- inputs
def _gen(case, seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 100003 + case["id"])


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _rand(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def _keys(g, n, H, D):
    """Keys: a common direction for each head and a few wide channels, as projections of normalised activations have them."""
    x = _randn(g, n, H, D) + 0.5 * _randn(g, 1, H, D)
    x[..., 3::29] *= 4.0
    return x


def _values(g, n, H, D):
    return _randn(g, n, H, D) * torch.exp(0.4 * _randn(g, n, H, 1))


def _quantise(x, kept):
    """Codes and scales of rows [..., D]: scale = amax / Q, code = x ((1 / amax) Q) to the nearest."""
    x = x.float()
    if kept not in QMAX:
        return x.to(TORCH[kept]), None
    amax = x.abs().amax(-1)
    small = amax < TINY
    inv = torch.where(small, 0.0, (1.0 / torch.where(small, 1.0, amax)) * QMAX[kept])
    scale = torch.where(small, 0.0, amax / QMAX[kept])
    y = (x * inv.unsqueeze(-1)).clamp(-QMAX[kept], QMAX[kept])
    return (y.round() if kept == "int8" else y).to(TORCH[kept]), scale


def _layout(case, g):
    new, length, page = _list(case["new"]), _list(case["length"]), case["page"]
    S = len(new)
    need = [-(-n // page) for n in length]
    n_pages, width = sum(need) + 3, max(max(need), 1)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    pages = torch.zeros(S, width, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        pages[s, :n] = order[at:at + n]
        at += n
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    row_seq = torch.repeat_interleave(torch.arange(S, device="cuda"), torch.tensor(new, device="cuda"))
    start_t, length_t = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (start, length))
    row = torch.arange(start[-1], device="cuda")
    pos = length_t[row_seq].long() - start_t[row_seq + 1].long() + row
    return dict(S=S, T=start[-1], n_pages=n_pages, width=width, pages=pages, start=start_t, length=length_t, row_seq=row_seq, pos=pos, max_len=max(max(length), 1))


def _summarise(k):
    """Codes [..., 2, D] (largest, smallest) and scales [...] of keys [..., page, D] in 32 bits; NaN where a position does not count."""
    top = torch.where(torch.isnan(k), -math.inf, k).amax(-2)
    low = torch.where(torch.isnan(k), math.inf, k).amin(-2)
    both = torch.stack([top, low], -2)
    amax = both.abs().amax((-1, -2))
    small = amax < TINY
    inv = torch.where(small, 0.0, (1.0 / torch.where(small, 1.0, amax)) * 127.0)
    codes = (both * inv[..., None, None]).clamp(-127.0, 127.0).round().to(torch.int8)
    return codes, torch.where(small, 0.0, amax / 127.0)


def _pool(g, st, case, topics=False):
    """Key and value pools; with `topics` the pages' keys have directions of their own, and the summaries of all pages are made as well."""
    H, D, page, kept = case["kv_heads"], case["D"], case["page"], case["kept"]
    pool, summary = [], None
    if topics:
        summary = (torch.empty(st["n_pages"], H, 2, D, dtype=torch.int8, device="cuda"), torch.empty(st["n_pages"], H, dtype=torch.float32, device="cuda"))
    for make in (_keys, _values):
        codes = torch.empty(st["n_pages"], H, page, D, dtype=TORCH[kept], device="cuda")
        scale = torch.empty(st["n_pages"], H, page, dtype=torch.float32, device="cuda") if kept in QMAX else None
        step = max(1, (1 << 26) // (H * page * D))
        for a in range(0, st["n_pages"], step):
            n = min(step, st["n_pages"] - a)
            x = make(g, n * page, H, D).reshape(n, page, H, D).transpose(1, 2)
            if topics and make is _keys:
                x = x + 0.8 * _randn(g, n, H, 1, D)
            c, sc = _quantise(x.to(TORCH[case["dtype"]]), kept)
            codes[a:a + n] = c
            if scale is not None:
                scale[a:a + n] = sc
            if topics and make is _keys:
                y = c.float() if sc is None else c.float() * sc.unsqueeze(-1)
                summary[0][a:a + n], summary[1][a:a + n] = _summarise(y)
        pool += [codes, scale]
    return (pool[0], pool[2], pool[1], pool[3]), summary


def _pages_inputs(case, g):
    S, page, most = case["S"], case["page"], case["most"]
    a = _rand(g, most // 12 + 1, most, S)                            # lengths before
    if case["change"] == "round":
        # of eight drafted tokens and a correction some are kept, the next nine are to be written
        rows0 = rows1 = torch.full((S,), 9, dtype=torch.int32, device="cuda")
        b = a + _rand(g, 1, 10, S)
    else:
        u = torch.rand(S, generator=g, device="cuda")
        comes, ends = u < 0.125, u > 0.875
        a = torch.where(comes, 0, a)
        b = torch.where(comes, _rand(g, most // 3 + 1, most, S), torch.where(ends, 0, a + 1))
        rows0, rows1 = torch.ones_like(a), torch.where(comes, b, 1)
    need = lambda x: int(((x + page - 1) // page).sum())            # noqa: E731
    n0, n1 = need(a), need(b)
    n_pages = n0 + max(0, n1 - n0) // 2 + 1 if case["tight"] else n0 + n1 + 8
    width = (most + 10 + page - 1) // page + 1
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    T = 9 * S + 5 if case["change"] == "round" else S * most // 10 + 2 * S + 9           # room for the rows of a call
    state = dict(pages=torch.zeros(S, width, dtype=torch.int32, device="cuda"), held=torch.zeros(S, dtype=torch.int32, device="cuda"),
                 borrowed=torch.zeros(S, dtype=torch.int32, device="cuda"), free=order, n_free=torch.full((1,), n_pages, dtype=torch.int32, device="cuda"))
    st = dict(S=S, T=T, n_pages=n_pages, width=width, table=state, before=(a, rows0), after=(b.to(torch.int32), rows1.to(torch.int32)))
    _plain_step(st, case, *st["before"])
    return st


def _rotary_inputs(case, g):
    st = _layout(case, g)
    H, D, T, dt, heads = case["kv_heads"], case["D"], st["T"], TORCH[case["dtype"]], case["heads"]
    x = torch.empty(T, heads + 2 * H, D, dtype=dt, device="cuda")    # a fused projection's rows
    x[:, :heads] = (1.2 * _randn(g, T, heads, D)).to(dt)
    x[:, heads:heads + H] = _keys(g, T, H, D).to(dt)
    x[:, heads + H:] = _values(g, T, H, D).to(dt)
    st.update(q=x[:, :heads], k=x[:, heads:heads + H], v=x[:, heads + H:])
    st["positions"] = st["axis"] = None
    if case["axes"] > 1:
        # frame, height, width (and one more) of what was kept, behind what came before
        st["positions"] = torch.stack([_rand(g, 0, 1 << 17, 1) + _rand(g, 0, 8 if a == 0 else 96, T).sort().values for a in range(case["axes"])]).contiguous()
        st["axis"] = (torch.arange(case["R"] // 2, device="cuda") % case["axes"]).to(torch.int32)
    if case["kind"] == "rotate_write":
        st["pool"], _ = _pool(g, st, case)
    return st


SCALING = {"plain": dict(), "linear": dict(factor=4.0), "base": dict(factor=8.0), "bands": dict(factor=8.0, original=8192, low=1.0, high=4.0),
           "ramp": dict(factor=16.0, original=4096, low=1.0, high=32.0)}
BASE = 500000.0


def _magnitude(case):
    return 0.1 * math.log(SCALING["ramp"]["factor"]) + 1.0 if case["scaling"] == "ramp" else 1.0


def _frequencies(case):
    """Angle from one position to the next, in 64 bits."""
    R, c = case["R"], SCALING[case["scaling"]]
    base = BASE * c["factor"] ** (R / (R - 2.0)) if case["scaling"] == "base" else BASE
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    f = base ** (-2.0 * i / R)
    if case["scaling"] == "linear":
        f = f / c["factor"]
    if case["scaling"] == "bands":
        turns = c["original"] * f / (2.0 * math.pi)                   # over the original context
        keep = ((turns - c["low"]) / (c["high"] - c["low"])).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / c["factor"])
    if case["scaling"] == "ramp":
        at = lambda turns: R * math.log(c["original"] / (turns * 2.0 * math.pi)) / (2.0 * math.log(BASE))       # noqa: E731
        lo, hi = max(math.floor(at(c["high"])), 0), min(math.ceil(at(c["low"])), R - 1)
        keep = 1.0 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / c["factor"])
    return f


def _sparse_inputs(case, g):
    st = _layout(case, g)
    st["pool"], st["summary"] = _pool(g, st, case, topics=True)
    T = st["T"]
    if case["kind"] == "summary":
        st["summary"][0].zero_()
        st["summary"][1].zero_()
        return st
    x = torch.empty(T, case["heads"] + 2 * case["kv_heads"], case["D"], dtype=TORCH[case["dtype"]], device="cuda")
    x[:] = 1.2 * _randn(g, *x.shape)
    st["q"], st["visible"] = x[:, :case["heads"]], None
    if case["tree"]:            # each token behind an earlier one, itself visible
        bits = []
        for n in _list(case["new"]):
            parent = torch.randint(0, 1 << 30, (n,), generator=g, device="cuda").tolist()
            seen = []
            for i in range(n):
                seen.append((seen[parent[i] % i] if i else 0) | 1 << i)
            bits += seen
        st["visible"] = torch.tensor(bits, dtype=torch.int64, device="cuda")
    return st


def _inputs(case, seed):
    g = _gen(case, seed)
    make = {"pages": _pages_inputs, "rotate": _rotary_inputs, "rotate_write": _rotary_inputs, "summary": _sparse_inputs, "sparse": _sparse_inputs}[case["kind"]]
    return make(case, g)


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["kind"].startswith("rotate"):
        st["freq"] = _frequencies(case)
    if not own:
        return st
    import paper_2605_02218_amd as C
    DT = {"bf16": C.BF16, "fp16": C.FP16, "int8": C.INT8, "e4m3": C.E4M3}
    if case["kind"] == "pages":
        st["p"] = C.PagesParams(n_seq=st["S"], n_tokens=st["T"], page_size=case["page"], n_pages=st["n_pages"], max_pages=st["width"])
        t = st["table"]
        st["state"] = (t["pages"], t["held"], t["borrowed"], t["free"], t["n_free"])
        st["ws"] = torch.empty(C.pages_workspace_size(st["p"]) + 256, dtype=torch.uint8, device="cuda")
        return st
    p = C.CacheParams(n_seq=st["S"], n_tokens=st["T"], n_kv_heads=case["kv_heads"], head_dim=case["D"], page_size=case["page"],
                      n_pages=st["n_pages"], max_pages=st["width"], dtype=DT[case["dtype"]], cache_dtype=DT[case["kept"]])
    st["cache_p"] = p
    if case["kind"].startswith("rotate"):
        st["p"] = C.RotaryParams(n_seq=st["S"], n_tokens=st["T"], n_heads=case["heads"], n_kv_heads=case["kv_heads"], head_dim=case["D"], rotary_dim=case["R"],
                                 interleaved=case["interleaved"], n_axes=case["axes"], dtype=DT[case["dtype"]], magnitude=_magnitude(case))
        kind = {"plain": C.ROTARY_PLAIN, "linear": C.ROTARY_LINEAR, "base": C.ROTARY_BASE, "bands": C.ROTARY_BANDS, "ramp": C.ROTARY_RAMP}[case["scaling"]]
        st["steps"] = C.rotary_steps(case["R"], base=BASE, scaling=kind, **SCALING[case["scaling"]])
    if case["kind"] == "sparse":
        st["p"] = C.SparseParams(attend=C.AttendParams(cache=p, n_heads=case["heads"], max_len=st["max_len"], scale=1.0 / math.sqrt(case["D"])), top=case["top"],
                                 first=case["first"], recent=case["recent"])
        st["ws"] = torch.empty(C.sparse_workspace_size(st["p"]) + 256, dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if own:
        import paper_2605_02218_amd as C
        if case["kind"] == "pages":
            # to the lengths after and back to those before, which undoes it
            there = C.pages_step(st["p"], st["state"], *st["after"], workspace=st["ws"])
            back = C.pages_step(st["p"], st["state"], *st["before"], workspace=st["ws"])
            return {"there": there._asdict(), "back": back._asdict(), "table": _table(st)}
        if case["kind"] == "rotate":
            q, k = C.rotate(st["p"], st["q"], st["k"], st["steps"], st["start"], st["length"], positions=st["positions"], axis=st["axis"])
            return {"q": q, "k": k}
        if case["kind"] == "rotate_write":
            q = C.rotate_write(st["p"], st["cache_p"], st["q"], st["k"], st["v"], st["steps"], st["start"], st["length"], st["pages"], st["pool"],
                               positions=st["positions"], axis=st["axis"])
            return dict(_kept(st["pool"]), q=q)
        C.block_summary(st["cache_p"], st["start"], st["length"], st["pages"], st["pool"], st["summary"])
        made = {"summary": st["summary"][0], "summary_scale": st["summary"][1]}
        if case["kind"] == "summary":
            return made
        out, lse, blocks = C.sparse_attend(st["p"], st["q"], st["start"], st["length"], st["pages"], st["pool"], st["summary"], visible=st["visible"],
                                           workspace=st["ws"], want_lse=True)
        return dict(made, out=out, lse=lse, blocks=blocks)
    if case["kind"] == "pages":
        there, back = _plain_step(st, case, *st["after"]), _plain_step(st, case, *st["before"])
        return {"there": there, "back": back, "table": _table(st)}
    if case["kind"].startswith("rotate"):
        return _plain_rotary(st, case)
    made = _plain_summary(st, case)
    return made if case["kind"] == "summary" else dict(made, **_plain_sparse(st, case))


def _table(st):
    t = st["table"]
    return {"held": t["held"], "free": t["n_free"]}


def _kept(pool):
    return {n: t for n, t in zip(("k", "v", "k_scale", "v_scale"), pool) if t is not None}


def _plain_step(st, case, want, rows):
    """Pages given back, pages given out, and where the rows of the next call lie; all integers."""
    t, page, width, n_pages = st["table"], case["page"], st["width"], st["n_pages"]
    held, borrowed, table, free, n_free = (t[n].long() for n in ("held", "borrowed", "pages", "free", "n_free"))
    want = want.long().clamp_min(0)
    rows = torch.minimum(rows.long().clamp_min(0), want)
    need = (want + page - 1) // page
    fits = need <= width
    goal = torch.where(fits, need, held)
    keep = torch.maximum(goal, borrowed)
    gives = (held - keep).clamp_min(0)
    asks = (goal - held).clamp_min(0)
    R = gives.sum()
    there = n_free + R
    j = torch.arange(width, device="cuda")[None]
    # given back: the last page of the last sequence first, on top of the list
    order = (gives.cumsum(0) - gives)[:, None] + j - keep[:, None]
    back = (j >= keep[:, None]) & (j < held[:, None])
    ext = torch.cat([free, torch.zeros(1, dtype=torch.long, device="cuda")])
    ext = ext.scatter(0, torch.where(back, n_free + R - 1 - order, n_pages).reshape(-1), table.reshape(-1))
    # given out, from the top, in the order of the sequences, none of which overtakes another
    served = (asks.cumsum(0) <= there) | (asks == 0)
    ok = served & fits
    order = (asks.cumsum(0) - asks)[:, None] + j - held[:, None]
    out = (j >= held[:, None]) & (j < goal[:, None]) & served[:, None]
    table = torch.where(out, ext[torch.where(out, there - 1 - order, n_pages)], table)
    held = torch.where(served, torch.where(goal < held, goal, torch.maximum(goal, held)), held)
    t["pages"].copy_(table)
    t["free"].copy_(ext[:n_pages])
    t["n_free"].copy_(there - (asks * served).sum())
    t["held"].copy_(held)
    t["borrowed"].copy_(torch.minimum(borrowed, held))
    n = torch.where(ok, rows, 0)
    room = (n.cumsum(0) <= st["T"]) | (n == 0)
    n = torch.where(room, n, 0)
    start = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), n.cumsum(0)])
    length = torch.where(ok & room, want, torch.minimum(want - rows, held * page))
    row = torch.arange(st["T"], device="cuda")
    s = torch.searchsorted(start, row, right=True) - 1
    real = row < start[-1]
    safe = s.clamp_max(st["S"] - 1)
    pos = length[safe] - start[safe + 1] + row
    slot = table[safe, torch.where(real, pos // page, 0)] * page + pos % page
    i32 = torch.int32
    return {"start": start.to(i32), "length": length.to(i32), "outcome": torch.where(ok, torch.where(room, 0, 2), 1).to(i32),
            "slots": torch.where(real, slot, -1), "positions": torch.where(real, pos, -1).to(i32)}


def _turned(x, c, s, R, interleaved):
    """Rows [T, H, D] in 32 bits, their first R elements turned."""
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
    u, v = a * c - b * s, b * c + a * s
    y = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([y, x[..., R:]], -1)


def _angles(st, case):
    pos = st["pos"][:, None] if st["positions"] is None else st["positions"][st["axis"].long()].t()
    return pos.double() * st["freq"]


def _plain_rotary(st, case):
    angle = _angles(st, case)
    c, s = ((f(angle) * _magnitude(case)).float()[:, None] for f in (torch.cos, torch.sin))
    dt = TORCH[case["dtype"]]
    q = _turned(st["q"].float(), c, s, case["R"], case["interleaved"]).to(dt)
    k = _turned(st["k"].float(), c, s, case["R"], case["interleaved"])
    if case["kind"] == "rotate":
        return {"q": q, "k": k.to(dt)}
    p, at = st["pages"][st["row_seq"], st["pos"] // case["page"]].long(), st["pos"] % case["page"]
    for x, codes, scale in ((k, st["pool"][0], st["pool"][2]), (st["v"], st["pool"][1], st["pool"][3])):
        y, sc = _quantise(x, case["kept"])
        if scale is None:
            codes[p, :, at] = y
        else:
            codes.view(torch.uint8)[p, :, at] = y.view(torch.uint8)
            scale[p, :, at] = sc
    return dict(_kept(st["pool"]), q=q)


def _gathered(codes, scale, *at):
    """Rows of the pool in 32 bits."""
    if scale is None:
        return codes[at].float()
    return codes.view(torch.uint8)[at].view(codes.dtype).float() * scale[at].unsqueeze(-1)


def _plain_summary(st, case):
    """Summaries of the pages that hold rows of the batch."""
    page = case["page"]
    first = torch.ones(st["T"], dtype=torch.bool, device="cuda")        # rows that are the first of theirs on a page
    first[1:] = (st["row_seq"][1:] != st["row_seq"][:-1]) | (st["pos"][1:] % page == 0)
    s, b = st["row_seq"][first], st["pos"][first] // page
    id = st["pages"][s, b].long()
    k = _gathered(st["pool"][0], st["pool"][2], id)
    at = b[:, None] * page + torch.arange(page, device="cuda")
    k = torch.where((at < st["length"][s].long()[:, None])[:, None, :, None], k, math.nan)
    st["summary"][0][id], st["summary"][1][id] = _summarise(k)
    return {"summary": st["summary"][0], "summary_scale": st["summary"][1]}


def _chosen(st, case):
    """[T, H, top] blocks of each row and key head, ascending, -1 behind the last.  Scores are sums of whole numbers below 2^24, then two roundings."""
    H, D, page, G = case["kv_heads"], case["D"], case["page"], case["heads"] // case["kv_heads"]
    T, top, first, recent = st["T"], case["top"], case["first"], case["recent"]
    q, sq = _quantise(st["q"], "int8")
    q = q.float().reshape(T, H, G, D)
    q = torch.cat([q.clamp_min(0.0), q.clamp_max(0.0)], -1)
    nb_all = st["width"]
    id = st["pages"].long()[st["row_seq"]]                              # [T, nb]
    M = st["summary"][0][id].float().permute(0, 2, 3, 4, 1).reshape(T, H, 2 * D, nb_all)
    z = torch.matmul(q, M)                                              # [T, H, G, nb]
    z = z * st["summary"][1][id].permute(0, 2, 1).unsqueeze(2)
    z = (z * sq.reshape(T, H, G, 1)).amax(2)
    hi = st["length"][st["row_seq"]].long() if case["tree"] else st["pos"] + 1
    nb = ((hi + page - 1) // page)[:, None, None]
    b = torch.arange(nb_all, device="cuda")[None, None]
    z = torch.where((b < first) | (b >= nb - recent), math.inf, z)
    z = torch.where(b < nb, z, -math.inf)
    best = torch.sort(z, dim=-1, descending=True, stable=True)
    best = torch.where(best.values > -math.inf, best.indices, nb_all)[..., :top]
    if nb_all < top:
        best = torch.cat([best, torch.full((T, H, top - nb_all), nb_all, device="cuda")], -1)
    best = best.sort(-1).values
    return torch.where(best < nb_all, best, -1)


def _plain_sparse(st, case):
    H, D, page, G = case["kv_heads"], case["D"], case["page"], case["heads"] // case["kv_heads"]
    T, top = st["T"], case["top"]
    k, v, ks, vs = st["pool"]
    blocks = _chosen(st, case)
    id = st["pages"].long()[st["row_seq"][:, None, None], blocks.clamp_min(0)]
    h = torch.arange(H, device="cuda")[None, :, None]
    j = blocks.unsqueeze(-1) * page + torch.arange(page, device="cuda")                   # [T, H, top, page]
    old = (st["length"] - (st["start"][1:] - st["start"][:-1])).long()[st["row_seq"]][:, None, None, None]
    if case["tree"]:
        bit = (st["visible"][:, None, None, None] >> (j - old).clamp(0, 63)) & 1
        seen = (j < old) | ((bit != 0) & (j - old < 64))
    else:
        seen = j <= st["pos"][:, None, None, None]
    seen = (seen & (blocks >= 0).unsqueeze(-1)).reshape(T, H, 1, top * page)
    K = _gathered(k, ks, id, h).reshape(T, H, top * page, D)
    z = torch.matmul(st["q"].float().reshape(T, H, G, D), K.transpose(2, 3)) * (1.0 / math.sqrt(D))
    del K
    z = z.masked_fill_(~seen, -math.inf)
    m = z.amax(-1, keepdim=True).clamp_min(-3e38)
    z = z.sub_(m).exp_()
    total = z.sum(-1, keepdim=True)
    o = torch.matmul(z, _gathered(v, vs, id, h).reshape(T, H, top * page, D)) / total.clamp_min(1e-38)
    lse = (m + total.log()).squeeze(-1)
    return {"out": o.reshape(T, H * G, D).to(TORCH[case["dtype"]]), "lse": lse.reshape(T, H * G), "blocks": blocks.to(torch.int32)}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "pages":
        S, page = case["S"], case["page"]
        rows = 18.0 * S if case["change"] == "round" else S * (case["most"] / 12.0 + 2.0)
        moved = S * 9.0 / page if case["change"] == "round" else S * case["most"] / (4.0 * page)
        # per row a place and a position; per page one entry in, one out; per sequence and call what is asked for, the state, the answer
        return {"bytes": 12.0 * rows + 16.0 * moved + 2.0 * 36.0 * S, "flops": rows}
    e, kept = SIZE[case["dtype"]], SIZE[case["kept"]]
    new, length = _list(case["new"]), _list(case["length"])
    H, D, heads, T, page = case["kv_heads"], case["D"], case["heads"], sum(new), case["page"]
    row = D * kept + (4.0 if case["kept"] in QMAX else 0.0)              # a token's key of one head in the cache
    if case["kind"].startswith("rotate"):
        by = 2.0 * T * (heads + H) * D * e if case["kind"] == "rotate" else T * (2.0 * heads * D * e + 2.0 * H * (D * e + row))
        return {"bytes": by, "flops": 3.0 * T * (heads + H) * case["R"]}
    by = fl = 0.0
    for n, m in zip(new, length):
        if n == 0:
            continue
        touched = (m - 1) // page - (m - n) // page + 1
        by += H * ((m - (m - n) // page * page) * row + touched * (2.0 * D + 4.0))
        fl += 2.0 * (m - (m - n) // page * page) * H * D
        if case["kind"] == "summary":
            continue
        nb = -(-m // page)
        seen = min(min(nb, case["top"]) * page, m)
        by += H * (nb * (2.0 * D + 4.0) + 2.0 * seen * row) + n * heads * (2.0 * D * e + 4.0) + 4.0 * n * H * case["top"]
        fl += n * heads * (4.0 * D * nb + 4.0 * D * seen)
    return {"bytes": by, "flops": fl}


# ---------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    if case["kind"] in ("pages", "summary"):
        return None             # whole numbers, and scales that are one division
    st = _inputs(case, seed)
    return _exact_rotary(st, case) if case["kind"].startswith("rotate") else _exact_sparse(st, case)


def _exact_rotary(st, case):
    R, D, dev = case["R"], case["D"], "cuda"
    first = torch.empty(R // 2, dtype=torch.long, device=dev)            # the pairs' elements
    if case["interleaved"]:
        first = 2 * torch.arange(R // 2, device=dev)
        second = first + 1
    else:
        first = torch.arange(R // 2, device=dev)
        second = first + R // 2
    f = _frequencies(case)
    mag = _magnitude(case)

    def turn(x):
        y = x.double().clone()
        for i in range(R // 2):
            pos = st["pos"] if st["positions"] is None else st["positions"][int(st["axis"][i])]
            w = torch.polar(torch.full((x.shape[0], 1), mag, dtype=torch.float64, device=dev), (pos.double() * f[i])[:, None])
            z = torch.complex(x[:, :, first[i]].double(), x[:, :, second[i]].double()) * w
            y[:, :, first[i]], y[:, :, second[i]] = z.real, z.imag
        return y

    q, k = turn(st["q"]), turn(st["k"])
    if case["kind"] == "rotate":
        return {"q": q, "k": k}
    res = {"q": q}
    for name, x, codes, scale in (("k", k, st["pool"][0], st["pool"][2]), ("v", st["v"].double(), st["pool"][1], st["pool"][3])):
        whole, sc = codes.double(), None if scale is None else scale.double()
        row = 0
        for s, (n, m) in enumerate(zip(_list(case["new"]), _list(case["length"]))):
            pos = torch.arange(m - n, m, device=dev)
            slot, at = st["pages"][s, pos // case["page"]].long(), pos % case["page"]
            rows = x[row:row + n]
            row += n
            if scale is not None:
                top = rows.abs().amax(-1)
                sc[slot, :, at] = top / 448.0
                rows = rows / top[..., None] * 448.0
                # to the nearest value of four bits of significand, subnormal below 2^-6
                step = torch.exp2(torch.floor(torch.log2(rows.abs().clamp_min(2.0 ** -6))) - 3)
                rows = torch.round(rows / step) * step
            whole[slot, :, at] = rows
        res[name] = whole
        if scale is not None:
            res[name + "_scale"] = sc
    return res


def _exact_sparse(st, case):
    """The choice is that of whole numbers; the attention over it row by row."""
    _plain_summary(st, case)
    blocks = _chosen(st, case).tolist()
    new, length, page, H, D = _list(case["new"]), _list(case["length"]), case["page"], case["kv_heads"], case["D"]
    if sum(new) * H > 1600:
        return None
    G, c = case["heads"] // H, D ** -0.5
    k, v, ks, vs = st["pool"]
    table = st["pages"].tolist()
    out = torch.zeros(st["T"], case["heads"], D, dtype=torch.float64, device="cuda")
    lse = torch.full((st["T"], case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    t = 0
    for s, (n, m) in enumerate(zip(new, length)):
        for i in range(n):
            bits = int(st["visible"][t]) if case["tree"] else 0
            for h in range(H):
                picked = [b for b in blocks[t][h] if b >= 0]
                id = torch.tensor([table[s][b] for b in picked], device="cuda")
                j = (torch.tensor(picked, device="cuda")[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)
                K, V = k[id, h].double(), v[id, h].double()
                if ks is not None:
                    K, V = K * ks[id, h].double().unsqueeze(-1), V * vs[id, h].double().unsqueeze(-1)
                K, V = K.reshape(-1, D), V.reshape(-1, D)
                if case["tree"]:
                    sees = torch.tensor([bits >> b & 1 == 1 for b in range(n)], device="cuda")
                    seen = (j < m - n) | ((j >= m - n) & (j < m) & sees[(j - (m - n)).clamp(0, n - 1)])
                else:
                    seen = j <= m - n + i
                z = c * (st["q"][t, h * G:(h + 1) * G].double() @ K[seen].t())
                lse[t, h * G:(h + 1) * G] = torch.logsumexp(z, 1)
                out[t, h * G:(h + 1) * G] = torch.softmax(z, 1) @ V[seen]
            t += 1
    return {"summary": None, "summary_scale": None, "out": out, "lse": lse, "blocks": None}
