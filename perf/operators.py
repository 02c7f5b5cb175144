"""Timed cases of what surrounds the verification of a drafted segment: new tokens into a paged key / value cache and back out of
it, their attention over the cache, and penalties, biases and masks on their logits.

listed() are the fixed cases, draw() gives more of the same ranges.  prepare() makes a program's inputs; run() is one pass, in
plain torch operations, or through the library's entry points where `own` is true; exact() is what the outputs are in 64 bits.

A batch is described the way the entry points take it: rows start[s] .. start[s + 1] - 1 of the packed tensors are the last
positions of sequence s, length[s] is its length with them, pages[s] are the pages that hold it.
"""
import math

import torch

own = False

TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
QMAX = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100          # rows without an element that large are stored as zeros


def listed():
    return [
        # one interactive sequence of a small draft model, one token: a single short call in a chain of them
        attend("attend_token", 1, [1], [1500], 16, 2, 64, 16, "bf16", "bf16"),
        # a full decoding batch of the target, one token each, 8-bit cache
        attend("attend_decode", 2, [1] * 64, _spread(64, 700, 7900), 32, 8, 128, 64, "bf16", "e4m3"),
        # verification: eight drafted tokens of each of 32 sequences
        attend("attend_verify", 3, [8] * 32, _spread(32, 900, 6100), 64, 8, 128, 64, "bf16", "bf16"),
        # a drafted tree of eleven tokens behind one very long context
        attend("attend_long", 4, [11], [120001], 32, 4, 128, 128, "fp16", "int8", tree=True),
        # prompts: 2880 image tokens and 128 words each, nothing cached before
        attend("attend_prompt", 5, [3008] * 4, [3008] * 4, 64, 8, 128, 64, "bf16", "bf16"),
        # a mixed batch of prompt chunks and single tokens with a sliding window, a draft model's heads
        attend("attend_chunks", 6, [1, 517, 1100, 1, 64], [4001, 5200, 2300, 77, 9001], 32, 32, 96, 16, "fp16", "e4m3", window=2048),
        # prompts of a batch into an 8-bit cache
        cache("write_prompt", "write", 7, [3008] * 8, [3008] * 8, 8, 128, 64, "bf16", "e4m3"),
        # eight drafted tokens and the correction of a full batch
        cache("write_round", "write", 8, [9] * 64, _spread(64, 300, 2500), 8, 128, 16, "fp16", "int8"),
        # a batch's caches as dense tensors, to be moved to another machine
        cache("read_batch", "read", 9, _spread(16, 1500, 6000), _spread(16, 1500, 6000), 8, 128, 64, "bf16", "int8"),
        # the last tokens of a few sequences of odd lengths
        cache("read_odd", "read", 10, [1, 333, 64, 0, 77], [1, 700, 64, 0, 1001], 32, 96, 16, "fp16", "fp16"),
        # rows of a full verification batch over a 152 k vocabulary, with histories, biases and grammar masks
        logits("logits_batch", 11, 64, 8, 151936, "bf16", 4000, 64, True),
        # one interactive sequence
        logits("logits_one", 12, 1, 1, 32000, "fp32", 1200, 8, False),
    ]


def _spread(n, lo, hi):
    """n lengths between lo and hi, in no order."""
    return [lo + (i * 7919 + 13) % n * (hi - lo) // max(n - 1, 1) for i in range(n)]


def _text(values):
    return ",".join(str(v) for v in values)


def _list(text):
    return [int(v) for v in text.split(",")]


def attend(name, id, new, length, heads, kv_heads, D, page, dtype, kept, window=0, tree=False):
    c = dict(kind="attend", id=id, new=_text(new), length=_text(length), heads=heads, kv_heads=kv_heads, D=D, page=page, dtype=dtype, kept=kept,
             window=window, tree=tree)
    return dict(c, name=name) if name else c


def cache(name, kind, id, new, length, kv_heads, D, page, dtype, kept):
    c = dict(kind=kind, id=id, new=_text(new), length=_text(length), kv_heads=kv_heads, D=D, page=page, dtype=dtype, kept=kept)
    return dict(c, name=name) if name else c


def logits(name, id, S, L, V, dtype, history, biased, masked):
    c = dict(kind="logits", id=id, S=S, L=L, V=V, dtype=dtype, history=history, biased=biased, masked=masked)
    return dict(c, name=name) if name else c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    u, id = rng.random(), rng.randint(100, 1 << 20)
    if u < 0.2:
        step = 8
        return logits(None, id, _log(rng, 1, 64), rng.randint(1, 8), step * _log(rng, 4000, 151936 // step), rng.choice(["bf16", "fp16", "fp32"])
                      if u < 0.1 else "bf16", _log(rng, 1, 8000) if u < 0.1 else _log(rng, 1, 4000), rng.choice([0, 3, 64, 300]), rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    kept = rng.choice([dtype, "int8", "e4m3"])
    D, page = rng.choice([64, 96, 128, 128]), rng.choice([16, 32, 64, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    S = _log(rng, 1, 64)
    if u < 0.45:
        top = max(1, 24000 // S)
        new = [_log(rng, 1, top) for _ in range(S)]
        length = [n + rng.choice([0, rng.randint(0, 2000)]) for n in new]
        return cache(None, "write" if u < 0.33 else "read", id, new, length, min(kv_heads, 8), D, page, dtype, kept)
    heads = kv_heads * rng.choice([1, 2, 4, 5, 8])
    if u < 0.8:             # tokens and drafted segments
        n = rng.choice([1, 1, rng.randint(2, 16)])
        top = max(200, 1100000 // (S * max(kv_heads, 4)))          # as many bytes as the listed batch
        length = [n + _log(rng, 100, min(top, 120000)) for _ in range(S)]
        return attend(None, id, [n] * S, length, min(heads, 64), kv_heads, D, page, dtype, kept, rng.choice([0, 0, 0, 1024]) if n == 1 else 0, n > 1 and rng.random() < 0.3)
    S = min(S, 6)           # prompts and chunks of them
    heads = min(heads, 8 * kv_heads, 32 if kv_heads <= 32 else kv_heads)
    new = [_log(rng, 17, 1500) for _ in range(S)]
    length = [n + rng.choice([0, rng.randint(0, 2000)]) for n in new]
    return attend(None, id, new, length, heads, kv_heads, D, page, dtype, kept, rng.choice([0, 0, 512]))


# ---------------------------------------------------------------- inputs
def _gen(case, seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 100003 + case["id"])


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _keys(g, n, H, D):
    """Keys: a common direction for each head and a few wide channels, as projections of normalised activations have them."""
    x = _randn(g, n, H, D) + 0.5 * _randn(g, 1, H, D)
    x[..., 3::29] *= 4.0
    return x


def _values(g, n, H, D):
    return _randn(g, n, H, D) * torch.exp(0.4 * _randn(g, n, H, 1))


def _quantise(x, kept):
    """Codes and scales of rows [..., D]: scale = amax / Q, code = x (Q / amax) to the nearest."""
    x = x.float()
    if kept not in QMAX:
        return x.to(TORCH[kept]), None
    amax = x.abs().amax(-1)
    small = amax < TINY
    inv = torch.where(small, 0.0, QMAX[kept] / torch.where(small, 1.0, amax))
    scale = torch.where(small, 0.0, amax / QMAX[kept])
    y = x * inv.unsqueeze(-1)
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
    return dict(new=new, len=length, S=S, T=start[-1], starts=start, n_pages=n_pages, width=width, pages=pages,
                start=torch.tensor(start, dtype=torch.int32, device="cuda"), length=torch.tensor(length, dtype=torch.int32, device="cuda"))


def _slots(st, page, S, pages, new, length):
    """Pool page and place in it of every row of the batch, in row order."""
    where = [torch.arange(n, device="cuda") + (length[s] - n) for s, n in enumerate(new)]
    p = torch.cat([pages[s][w // page] for s, w in enumerate(where)]).long()
    return p, torch.cat(where) % page


def _pool(g, st, case):
    """Key and value pools, everything in them made by the tokens of the sequences (or of earlier ones)."""
    H, D, page, kept = case["kv_heads"], case["D"], case["page"], case["kept"]
    out = []
    for make in (_keys, _values):
        codes = torch.empty(st["n_pages"], H, page, D, dtype=TORCH[kept], device="cuda")
        scale = torch.empty(st["n_pages"], H, page, dtype=torch.float32, device="cuda") if kept in QMAX else None
        step = max(1, (1 << 25) // (H * page * D))
        common = None
        for a in range(0, st["n_pages"], step):
            n = min(step, st["n_pages"] - a)
            x = make(g, n * page, H, D).to(TORCH[case["dtype"]])
            c, sc = _quantise(x.reshape(n, page, H, D).transpose(1, 2), kept)
            codes[a:a + n] = c
            if scale is not None:
                scale[a:a + n] = sc
        out += [codes, scale]
    return out[0], out[2], out[1], out[3]


def _inputs(case, seed):
    g = _gen(case, seed)
    if case["kind"] == "logits":
        return _logit_inputs(case, g)
    st = _layout(case, g)
    H, D, T, dt = case["kv_heads"], case["D"], st["T"], TORCH[case["dtype"]]
    if case["kind"] == "write":
        # keys and values as they leave a fused projection: columns of one wide row for each token
        x = torch.empty(T, 4 * H, D, dtype=dt, device="cuda")
        x[:, 2 * H:3 * H] = _keys(g, T, H, D).to(dt)
        x[:, 3 * H:] = _values(g, T, H, D).to(dt)
        st.update(k=x[:, 2 * H:3 * H], v=x[:, 3 * H:], pool=_pool(g, st, case))
        return st
    st["pool"] = _pool(g, st, case)
    if case["kind"] == "attend":
        st["q"] = (1.2 * _randn(g, T, case["heads"], D)).to(dt)
        st["visible"] = None
        if case["tree"]:        # each token behind an earlier one, itself visible
            bits = []
            for n in st["new"]:
                parent = torch.randint(0, 1 << 30, (n,), generator=g, device="cuda").tolist()
                seen = []
                for i in range(n):
                    seen.append((seen[parent[i] % i] if i else 0) | 1 << i)
                bits += [b - (1 << 64) if b >> 63 else b for b in seen]
            st["visible"] = torch.tensor(bits, dtype=torch.int64, device="cuda")
    return st


def _logit_inputs(case, g):
    S, L, V, dt = case["S"], case["L"], case["V"], TORCH[case["dtype"]]
    z = (2.0 * _randn(g, S, L, V)).to(dt)
    # text: few words make up most of a history
    n = [max(0, case["history"] - (s * 37) % max(1, case["history"] // 3)) for s in range(S)]
    start = [0]
    for m in n:
        start.append(start[-1] + m)
    words = (V * torch.rand(start[-1], generator=g, device="cuda") ** 4).to(torch.int32).clamp_(0, V - 1)
    drafted = (V * torch.rand(S, L, generator=g, device="cuda") ** 4).to(torch.int32).clamp_(0, V - 1)
    prompt = torch.tensor([m // 2 for m in n], dtype=torch.int32, device="cuda")
    u = torch.rand(S, 4, generator=g, device="cuda")
    penalties = torch.stack([1.0 + 0.3 * u[:, 0], 0.5 * u[:, 1], 0.2 * u[:, 2], 0.6 + 0.6 * u[:, 3]], 1).contiguous()
    m = case["biased"]
    bias = None
    if m:
        token = torch.stack([torch.randperm(V, generator=g, device="cuda")[:m] for _ in range(S)]).to(torch.int32).reshape(-1)
        bias = (torch.arange(0, S * m + 1, m, dtype=torch.int32, device="cuda"), token.contiguous(), 3.0 * _randn(g, S * m))
    allowed = None
    if case["masked"]:
        # a grammar allows anything in most states and a few words in others
        bits = torch.randint(-(1 << 31), 1 << 31, (S, L, (V + 31) // 32), generator=g, device="cuda")
        more = torch.randint(-(1 << 31), 1 << 31, (S, L, (V + 31) // 32), generator=g, device="cuda")
        few = (torch.rand(S, L, 1, generator=g, device="cuda") < 0.3)
        allowed = torch.where(few, bits & more, bits | more).to(torch.int32)
    return dict(z=z, words=words, start=torch.tensor(start, dtype=torch.int32, device="cuda"), starts=start, prompts=[m // 2 for m in n], prompt=prompt,
                drafted=drafted, penalties=penalties, bias=bias, allowed=allowed)


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if not own:
        return st
    import paper_2605_02218_amd as C
    DT = {"fp32": C.FP32, "bf16": C.BF16, "fp16": C.FP16, "int8": C.INT8, "e4m3": C.E4M3}
    if case["kind"] == "logits":
        st["p"] = C.LogitsParams(n_seq=case["S"], n_pos=case["L"], vocab=case["V"], dtype=DT[case["dtype"]])
        st["out"] = torch.empty_like(st["z"])
        return st
    p = C.CacheParams(n_seq=st["S"], n_tokens=st["T"], n_kv_heads=case["kv_heads"], head_dim=case["D"], page_size=case["page"],
                      n_pages=st["n_pages"], max_pages=st["width"], dtype=DT[case["dtype"]], cache_dtype=DT[case["kept"]])
    st["p"] = p
    if case["kind"] == "attend":
        st["p"] = C.AttendParams(cache=p, n_heads=case["heads"], max_len=max(st["len"]), window=case["window"], scale=1.0 / math.sqrt(case["D"]))
        st["ws"] = torch.empty(C.attend_workspace_size(st["p"]) + 256, dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if own:
        import paper_2605_02218_amd as C
        if case["kind"] == "logits":
            return C.adjust_logits(st["p"], st["z"], st["words"], st["start"], st["penalties"], prompt_len=st["prompt"], drafted=st["drafted"],
                                   bias=st["bias"], allowed=st["allowed"], out=st["out"])
        if case["kind"] == "write":
            C.cache_write(st["p"], st["k"], st["v"], st["start"], st["length"], st["pages"], st["pool"])
            return _kept(st["pool"])
        if case["kind"] == "read":
            k, v = C.cache_read(st["p"], st["pool"], st["start"], st["length"], st["pages"])
            return {"k": k, "v": v}
        out, lse = C.attend(st["p"], st["q"], st["start"], st["length"], st["pages"], st["pool"], visible=st["visible"], workspace=st["ws"], want_lse=True)
        return {"out": out, "lse": lse}
    return {"logits": _plain_logits, "write": _plain_write, "read": _plain_read, "attend": _plain_attend}[case["kind"]](st, case)


def _kept(pool):
    return {n: t for n, t in zip(("k", "v", "k_scale", "v_scale"), pool) if t is not None}


def _plain_write(st, case):
    p, at = _slots(st, case["page"], st["S"], st["pages"], st["new"], st["len"])
    for x, codes, scale in ((st["k"], st["pool"][0], st["pool"][2]), (st["v"], st["pool"][1], st["pool"][3])):
        c, sc = _quantise(x, case["kept"])
        if scale is None:
            codes[p, :, at] = c
        else:
            codes.view(torch.uint8)[p, :, at] = c.view(torch.uint8)
            scale[p, :, at] = sc
    return _kept(st["pool"])


def _rows(codes, scale, p, at):
    """Rows of the pool in 32 bits, [n, H, D]."""
    if scale is None:
        return codes[p, :, at].float()
    return codes.view(torch.uint8)[p, :, at].view(codes.dtype).float() * scale[p, :, at].unsqueeze(-1)


def _plain_read(st, case):
    p, at = _slots(st, case["page"], st["S"], st["pages"], st["new"], st["len"])
    k, v, ks, vs = st["pool"]
    dt = TORCH[case["dtype"]]
    return {"k": _rows(k, ks, p, at).to(dt), "v": _rows(v, vs, p, at).to(dt)}


def _seen(case, n, length, visible):
    """[n, length]: which keys a row sees."""
    j = torch.arange(length, device="cuda")
    if visible is not None:
        old = length - n
        bit = (visible[:, None] >> (j - old).clamp(0, 63)[None]) & 1
        return (j < old)[None] | (bit != 0)
    pos = torch.arange(length - n, length, device="cuda")
    seen = j[None] <= pos[:, None]
    if case["window"]:
        seen &= j[None] > pos[:, None] - case["window"]
    return seen


def _plain_attend(st, case):
    k, v, ks, vs = st["pool"]
    H, D, page = case["kv_heads"], case["D"], case["page"]
    G = case["heads"] // H
    outs, lses = [], []
    for s, (n, length) in enumerate(zip(st["new"], st["len"])):
        if n == 0:
            continue
        a = st["starts"][s]
        need = -(-length // page)
        id = st["pages"][s, :need].long()

        def dense(codes, scale):
            x = codes.view(torch.uint8)[id].view(codes.dtype).float() if scale is not None else codes[id].float()
            if scale is not None:
                x = x * scale[id].unsqueeze(-1)
            return x.transpose(0, 1).reshape(H, need * page, D)[:, :length]

        K, V = dense(k, ks), dense(v, vs)
        q = st["q"][a:a + n].float().reshape(n, H, G, D).permute(1, 0, 2, 3).reshape(H, n * G, D)
        seen = _seen(case, n, length, None if st["visible"] is None else st["visible"][a:a + n]).repeat_interleave(G, 0)
        o, e = [], []
        step = max(1, (1 << 29) // (n * G * length))            # heads at a time: 2 GB of scores
        for h in range(0, H, step):
            z = torch.matmul(q[h:h + step], K[h:h + step].transpose(1, 2)) * (1.0 / math.sqrt(D))
            z = z.masked_fill_(~seen, -math.inf)
            m = z.amax(-1, keepdim=True).clamp_min(-3e38)
            z = z.sub_(m).exp_()
            total = z.sum(-1, keepdim=True)
            o.append(torch.matmul(z, V[h:h + step]) / total.clamp_min(1e-38))
            e.append((m + total.log()).squeeze(-1))
        outs.append(torch.cat(o).reshape(H, n, G, D).permute(1, 0, 2, 3).reshape(n, H * G, D).to(st["q"].dtype))
        lses.append(torch.cat(e).reshape(H, n, G).permute(1, 0, 2).reshape(n, H * G))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _plain_logits(st, case):
    S, L, V = case["S"], case["L"], case["V"]
    z = st["z"].float()
    said = torch.zeros(S, V, device="cuda")                      # generated so far
    asked = torch.zeros(S, V, device="cuda")                     # in the prompt
    for s in range(S):
        a, b = st["starts"][s], st["starts"][s + 1]
        w = st["words"][a:b].long()
        one = torch.ones(b - a, device="cuda")
        asked[s].index_add_(0, w[:st["prompts"][s]], one[:st["prompts"][s]])
        said[s].index_add_(0, w[st["prompts"][s]:], one[st["prompts"][s]:])
    rep, pres, freq, temp = (st["penalties"][:, i, None] for i in range(4))
    rows = []
    for t in range(L):
        x = z[:, t]
        x = torch.where((said + asked) > 0, torch.where(x > 0, x / rep, x * rep), x)
        rows.append(x - (freq * said + pres * (said > 0)))
        said = said.scatter_add(1, st["drafted"][:, t:t + 1].long(), torch.ones(S, 1, device="cuda"))
    x = torch.stack(rows, 1)
    if st["bias"] is not None:
        m = case["biased"]
        x.scatter_add_(2, st["bias"][1].long().reshape(S, 1, m).expand(S, L, m), st["bias"][2].reshape(S, 1, m).expand(S, L, m))
    x = x / temp.unsqueeze(-1)
    if st["allowed"] is not None:
        bit = torch.arange(32, device="cuda", dtype=torch.int32)
        ok = ((st["allowed"].unsqueeze(-1) >> bit) & 1).reshape(S, L, -1)[..., :V]
        x = x.masked_fill(ok == 0, -math.inf)
    return x.to(st["z"].dtype)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = {"fp32": 4.0, "bf16": 2.0, "fp16": 2.0, "int8": 1.0, "e4m3": 1.0}
    e = size[case["dtype"]]
    if case["kind"] == "logits":
        rows = case["S"] * case["L"]
        return {"bytes": rows * case["V"] * (2 * e + (0.125 if case["masked"] else 0.0)) + case["S"] * (4.0 * case["history"] + 8.0 * case["biased"] + 24.0),
                "flops": 4.0 * rows * case["V"]}
    new, length = _list(case["new"]), _list(case["length"])
    H, D = case["kv_heads"], case["D"]
    row = H * (D * size[case["kept"]] + (4.0 if case["kept"] in QMAX else 0.0))       # a token's keys in the cache
    if case["kind"] != "attend":
        return {"bytes": 2.0 * sum(new) * (row + H * D * e), "flops": 3.0 * sum(new) * H * D}
    by = fl = 0.0
    for n, m in zip(new, length):
        w = case["window"] or m
        first = max(0, m - n + 1 - w)                              # the first key that any row sees
        by += 2.0 * (m - first) * row + n * case["heads"] * (2.0 * D * e + 4.0)
        full = min(n, max(0, m - w))                               # rows with a whole window
        rest = n - full
        pairs = full * w + rest * (m - n) + rest * (rest + 1) / 2.0 if not case["tree"] else n * (m - n) + n * 3.0
        fl += 4.0 * D * case["heads"] * max(pairs, 0.0)
    return {"bytes": by, "flops": fl}


# ---------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    st = _inputs(case, seed)
    if case["kind"] == "logits":
        return _exact_logits(st, case)
    if case["kind"] == "write":
        return _exact_write(st, case)
    new, length, page, H, D = st["new"], st["len"], case["page"], case["kv_heads"], case["D"]
    k, v, ks, vs = st["pool"]
    table = st["pages"].tolist()

    def values(codes, scale, s, first, last):
        """Positions first .. last - 1 of sequence s in 64 bits, [H, n, D], page by page."""
        parts = []
        for b in range(first // page, -(-last // page)):
            lo, hi = max(first - b * page, 0), min(last - b * page, page)
            x = codes[table[s][b], :, lo:hi].to(torch.float64)
            parts.append(x if scale is None else x * scale[table[s][b], :, lo:hi, None].double())
        return torch.cat(parts, 1) if parts else torch.zeros(H, 0, D, dtype=torch.float64, device="cuda")

    if case["kind"] == "read":
        ends = [(s, m - n, m) for s, (n, m) in enumerate(zip(new, length))]
        return {"k": torch.cat([values(k, ks, *e).transpose(0, 1) for e in ends]), "v": torch.cat([values(v, vs, *e).transpose(0, 1) for e in ends])}
    if work(case)["flops"] > 3e12:
        return None
    G, c = case["heads"] // H, D ** -0.5
    out = torch.zeros(st["T"], case["heads"], D, dtype=torch.float64, device="cuda")
    lse = torch.full((st["T"], case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for s, (n, m) in enumerate(zip(new, length)):
        K, V = values(k, ks, s, 0, m), values(v, vs, s, 0, m)
        block = max(1, (1 << 27) // (m + 1))
        for i0 in range(0, n, block):
            i1 = min(n, i0 + block)
            hidden = torch.ones(i1 - i0, m, dtype=torch.bool, device="cuda")
            for i in range(i0, i1):
                pos, r = m - n + i, st["starts"][s] + i
                if st["visible"] is not None:
                    bits = int(st["visible"][r]) & ((1 << 64) - 1)
                    hidden[i - i0, :m - n] = False
                    for b in range(min(n, 64)):
                        if bits >> b & 1:
                            hidden[i - i0, m - n + b] = False
                else:
                    hidden[i - i0, max(0, pos + 1 - case["window"]) if case["window"] else 0:pos + 1] = False
            rows = slice(st["starts"][s] + i0, st["starts"][s] + i1)
            for h in range(case["heads"]):
                z = c * (st["q"][rows, h].double() @ K[h // G].t())
                z[hidden] = -math.inf
                lse[rows, h] = torch.logsumexp(z, 1)
                out[rows, h] = torch.softmax(z, 1) @ V[h // G]
    return {"out": out, "lse": lse}


def _exact_write(st, case):
    if case["kept"] == "int8":
        names = {"k": None, "v": None}
    else:
        names = {}
    res = {}
    for name, x, codes, scale in (("k", st["k"], st["pool"][0], st["pool"][2]), ("v", st["v"], st["pool"][1], st["pool"][3])):
        whole, sc = codes.double() if name not in names else None, None if scale is None else scale.double()
        x = x.double()
        for s, (n, m) in enumerate(zip(st["new"], st["len"])):
            pos = torch.arange(m - n, m, device="cuda")
            slot = st["pages"][s, pos // case["page"]].long()
            rows = x[st["starts"][s]:st["starts"][s + 1]]
            if scale is not None:
                top = rows.abs().amax(-1)
                sc[slot, :, pos % case["page"]] = top / QMAX[case["kept"]]
                rows = rows / top[..., None] * QMAX[case["kept"]]
            if whole is not None:
                if scale is not None:
                    # to the nearest value of four bits of significand, subnormal below 2^-6
                    step = torch.exp2(torch.floor(torch.log2(rows.abs().clamp_min(2.0 ** -6))) - 3)
                    rows = torch.round(rows / step) * step
                whole[slot, :, pos % case["page"]] = rows
        res[name] = whole
        if scale is not None:
            res[name + "_scale"] = sc
    return {n: res[n] for n in ("k", "v", "k_scale", "v_scale") if n in res}


def _exact_logits(st, case):
    S, L, V = case["S"], case["L"], case["V"]
    out = torch.empty(S, L, V, dtype=torch.float64, device="cuda")
    pen = st["penalties"].double().tolist()
    for s in range(S):
        w = st["words"][st["starts"][s]:st["starts"][s + 1]].long()
        r, p, f, T = pen[s]
        cut = st["prompts"][s]
        b = torch.zeros(V, dtype=torch.float64, device="cuda")
        if st["bias"] is not None:
            m = case["biased"]
            b[st["bias"][1][s * m:(s + 1) * m].long()] = st["bias"][2][s * m:(s + 1) * m].double()
        for t in range(L):
            mine = torch.cat([w[cut:], st["drafted"][s, :t].long()])
            n = torch.bincount(mine, minlength=V).double()
            any = torch.bincount(w[:cut], minlength=V) + n > 0
            x = st["z"][s, t].double()
            x = torch.where(any & (x > 0), x / r, torch.where(any, x * r, x))
            x = (x - f * n - p * (n > 0).double() + b) / T
            if st["allowed"] is not None:
                i = torch.arange(V, device="cuda")
                x[(st["allowed"][s, t][i // 32].long() >> (i % 32)) & 1 == 0] = -math.inf
            out[s, t] = x
    return out
