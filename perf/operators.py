"""Performance cases of the serving operators: rotary positions, the paged cache, attention over it, sampling.

A case names one call and its sizes; head layouts are those of keep_synth's decoders (28 query and 4 key/value heads, 40
and 8, the fp32 "tiny" one with 4 and 2) and a few generic ones, the vocabulary is theirs.  `run` computes a case in
elementary torch operations, or, where `own` is true, through the library.
"""
import math

import numpy as np
import torch

own = False

HEADS = {"7b": (28, 4, 128), "14b": (40, 8, 128), "tiny": (4, 2, 64), "small": (8, 2, 128), "narrow": (12, 12, 64),
         "wide": (8, 1, 256), "odd": (6, 3, 80)}
VOCAB = 152064
LIMIT = {"fp8": 448.0, "int8": 127.0}          # largest code of a cache format
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
WEIGHT_ONE = 2.0 ** 40                         # weight of a row's largest logit


def _rope(name, heads, rows, dtype, layout, rot, scaling="plain", top=40000):
    return {"name": name, "op": "rope", "heads": heads, "rows": rows, "dtype": dtype, "layout": layout, "rot": rot,
            "scaling": scaling, "top": top}


def _cache(name, heads, rows, dtype, fmt, page, spare=1.25):
    return {"name": name, "op": "cache", "heads": heads, "rows": rows, "dtype": dtype, "format": fmt, "page": page,
            "spare": spare}


def _attend(name, heads, seqs, new, ctx, dtype, fmt, page, window=0):
    """seqs sequences; new and ctx: (fewest, most) new tokens and earlier tokens of a sequence."""
    return {"name": name, "op": "attend", "heads": heads, "seqs": seqs, "new_lo": new[0], "new_hi": new[1],
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "dtype": dtype, "format": fmt, "page": page, "window": window}


def _sample(name, rows, vocab, dtype, top_k, top_p, min_p, mixed=False):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "top_k": top_k, "top_p": top_p,
            "min_p": min_p, "mixed": mixed}


def listed():
    return [
        # queries and keys of one decoded token: the smallest call, latency alone
        _rope("rope_token", "14b", 1, "bf16", "half", 128),
        # a layer's queries and keys of a whole 33k prompt, frequencies scaled by parts for a context four times as long
        _rope("rope_prompt", "14b", 33024, "bf16", "half", 128, "parts", 131072),
        # a chunk of a model that rotates neighbouring pairs of half a head, fp32 storage
        _rope("rope_part_f32", "7b", 1024, "f32", "interleaved", 64, "linear"),
        # one decoding step of 64 sequences: their new keys and values go into scattered pages, and come back
        _cache("cache_step_fp8", "14b", 64, "bf16", "fp8", 16),
        # one layer of a joined 33k prompt is stored in 8 bits and expanded again
        _cache("cache_prompt_int8", "14b", 33024, "bf16", "int8", 64),
        # the answer's next token over a joined 33k cache kept as it is
        _attend("attend_token_33k", "14b", 1, (1, 1), (33023, 33023), "bf16", "bf16", 64),
        # a decoding step of 64 ragged sequences over 8-bit pages
        _attend("attend_batch_fp8", "14b", 64, (1, 1), (0, 8191), "bf16", "fp8", 16),
        # the next 256-token instruction over a joined 33k cache kept in 8 bits
        _attend("attend_instr_int8", "14b", 1, (256, 256), (32768, 32768), "bf16", "int8", 64),
        # ragged chunks of eight prompts
        _attend("attend_chunks", "7b", 8, (100, 2000), (0, 16384), "bf16", "bf16", 32),
        # fp32 storage, a few new tokens of three short sequences, a sliding window, pages that end inside a tile
        _attend("attend_tiny_f32", "tiny", 3, (3, 65), (100, 1088), "f32", "f32", 20, 500),
        # one answer's next token
        _sample("sample_one", 1, VOCAB, "f32", 50, 0.9, 0.0),
        # the next tokens of a batch whose requests ask for different things
        _sample("sample_batch", 256, VOCAB, "f32", 0, 0.95, 0.02, True),
    ]


def draw(rng):
    """One more case of the ranges above; sizes log-uniform, odd ones included."""
    def logint(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    limit = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("rope", "cache", "attend", "sample")}
    while True:
        op = rng.choice(["rope", "cache", "attend", "attend", "sample"])
        heads = rng.choice(["7b", "14b", "7b", "14b", "tiny", "small", "narrow", "wide", "odd"])
        dtype = "f32" if heads in ("tiny", "odd") or rng.random() < 0.15 else "bf16"
        dh = HEADS[heads][2]
        fmt = rng.choice([dtype, "fp8", "int8"])
        page = rng.choice([1, 7, 16, 20, 32, 64, 100, 128, 256])
        if op == "rope":
            c = _rope("", heads, logint(1, 33024), dtype, rng.choice(["half", "interleaved"]),
                      rng.choice([dh, dh, dh // 2, 2 * rng.randint(1, dh // 2)]),
                      rng.choice(["plain", "linear", "base", "parts"]), logint(100, 1000000))
        elif op == "cache":
            c = _cache("", heads, logint(1, 33024), dtype, fmt, page)
        elif op == "attend":
            seqs = logint(1, 100)
            new = logint(1, 3000) if rng.random() < 0.5 else rng.randint(1, 4)
            ctx = logint(1, 40000)
            c = _attend("", heads, seqs, (max(1, new - rng.randrange(new)), new), (ctx - rng.randrange(ctx + 1), ctx),
                        dtype, fmt, page, logint(1, 4096) if rng.random() < 0.25 else 0)
        else:
            c = _sample("", logint(1, 256), rng.choice([VOCAB, logint(1, 300007)]), rng.choice(["f32", "f32", "bf16"]),
                        rng.choice([0, 1, logint(2, 2000)]), rng.choice([1.0, round(rng.uniform(0.1, 0.999), 3)]),
                        rng.choice([0.0, round(rng.uniform(0.001, 0.3), 3)]), rng.random() < 0.5)
        c.pop("name")
        if _cost(c) <= limit[op]:
            return c


# ---------------------------------------------------------------------------------------------------------------
# layouts (a function of the case alone, so that every seed has the same shapes)
# ---------------------------------------------------------------------------------------------------------------
def _lens(case):
    """(new tokens, all tokens) of each sequence"""
    r = np.random.Generator(np.random.PCG64(3))
    new = r.integers(case["new_lo"], case["new_hi"] + 1, size=case["seqs"])
    ctx = r.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=case["seqs"])
    return [int(v) for v in new], [int(a + b) for a, b in zip(new, ctx)]


def _pairs(case):
    """(visible (row, key) pairs, keys that some row sees), summed over the sequences"""
    pairs = keys = 0
    w = case["window"] or 1 << 60
    for n, total in zip(*_lens(case)):
        pos = np.arange(total - n, total, dtype=np.int64)
        pairs += int(np.minimum(pos + 1, w).sum())
        keys += total - max(0, total - n - w + 1)
    return pairs, keys


def _size(t):
    return torch.empty(0, dtype=TYPES[t]).element_size()


def _cost(case):
    if case["op"] == "attend":
        hq, hkv, dh = HEADS[case["heads"]]
        pages = sum(-(-t // case["page"]) for t in _lens(case)[1])
        rate = 1e12 if case["dtype"] == "bf16" else 1e11
        if 8 * hkv * dh * pages * case["page"] > 6 << 30:
            return math.inf                     # (the plain form's fp32 copies)
        return work(case)["flops"] / rate + work(case)["bytes"] / 5e12
    return work(case)["bytes"] / 5e12


def work(case):
    """Each input once, each output once; a key and its value once per key/value head."""
    if case["op"] == "rope":
        hq, hkv, dh = HEADS[case["heads"]]
        n = case["rows"] * (hq + hkv)
        return {"bytes": 2 * n * dh * _size(case["dtype"]) + 4 * case["rows"], "flops": 3 * n * case["rot"]}
    if case["op"] == "cache":
        _, hkv, dh = HEADS[case["heads"]]
        n = 2 * case["rows"] * hkv              # keys' and values' rows of one head
        code = n * (dh * _size(case["format"]) + (4 if case["format"] in LIMIT else 0))
        return {"bytes": 2 * n * dh * _size(case["dtype"]) + 2 * code + 8 * case["rows"], "flops": 3 * n * dh}
    if case["op"] == "attend":
        hq, hkv, dh = HEADS[case["heads"]]
        pairs, keys = _pairs(case)
        rows = sum(_lens(case)[0])
        code = 2 * keys * hkv * (dh * _size(case["format"]) + (4 if case["format"] in LIMIT else 0))
        return {"bytes": code + rows * hq * (2 * dh * _size(case["dtype"]) + 4), "flops": 4 * dh * hq * pairs}
    n = case["rows"] * case["vocab"]
    return {"bytes": n * _size(case["dtype"]) + 28 * case["rows"], "flops": 2 * n}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
SCALING = {"plain": (1.0, 0), "linear": (2.0, 0), "base": (4.0, 0), "parts": (4.0, 32768)}
THETA, FAST, SLOW = 1.0e6, 32.0, 1.0           # rotary base; turns over the trained length that bound the scaled parts


def _frequencies(case):
    """(angle per position of each pair, factor on the rotated values), in 64 bits"""
    rot, (factor, trained) = case["rot"], SCALING[case["scaling"]]
    j = np.arange(rot // 2, dtype=np.float64)
    base = THETA
    if case["scaling"] == "base" and rot > 2:
        base = THETA * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * j / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        turns = trained * f / (2.0 * math.pi)
        keep = np.clip((turns - SLOW) / (FAST - SLOW), 0.0, 1.0)
        return (1.0 - keep) * f / factor + keep * f, float(np.float32(0.1 * math.log(factor) + 1.0))
    return f, 1.0


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def ints(lo, hi, n):
        return torch.randint(lo, hi, (n,), generator=g, device="cuda", dtype=torch.int32)

    st = {"case": case}
    if case["op"] == "sample":
        rows, vocab, f32 = case["rows"], case["vocab"], torch.float32
        # logits as a decoder gives them: a broad bulk and a heavy upper tail
        x = 2.0 * normal(rows, vocab)
        x += 3.0 * torch.empty_like(x).exponential_(generator=g).sub_(3.0).clamp_(min=0.0)
        st["logits"] = x.to(TYPES[case["dtype"]])
        st["uniform"] = torch.rand(rows, generator=g, device="cuda")
        st["temperature"] = torch.full((rows,), 0.7, device="cuda")
        st["top_k"] = torch.full((rows,), case["top_k"], dtype=torch.int32, device="cuda")
        st["top_p"] = torch.full((rows,), case["top_p"], device="cuda")
        st["min_p"] = torch.full((rows,), case["min_p"], device="cuda")
        if case["mixed"]:       # requests that ask for other temperatures, for no cut or for the likeliest token
            st["temperature"] = (0.3 + 1.2 * torch.rand(rows, generator=g, device="cuda"))
            st["temperature"][ints(0, rows, max(1, rows // 16)).long()] = 0.0
            st["top_k"] = torch.where(ints(0, 3, rows) == 0, ints(1, 200, rows), st["top_k"])
            st["top_p"] = torch.where(ints(0, 4, rows) == 0, torch.ones(rows, device="cuda"), st["top_p"])
        st["tokens"] = torch.empty(rows, dtype=torch.int32, device="cuda")
        st["probs"] = torch.empty(rows, dtype=f32, device="cuda")
        if own:
            _own_sample_workspace(st)
        return st

    hq, hkv, dh = HEADS[case["heads"]]
    dtype = TYPES[case["dtype"]]
    if case["op"] == "rope":
        n = case["rows"]
        st["q"], st["k"] = normal(n, hq, dh).to(dtype), normal(n, hkv, dh).to(dtype)
        st["q_out"], st["k_out"] = torch.empty_like(st["q"]), torch.empty_like(st["k"])
        st["positions"] = torch.sort(ints(0, case["top"], n)).values
        f, st["magnitude"] = _frequencies(case)
        st["freq"] = torch.from_numpy(f).cuda()
        return st

    page, fmt = case["page"], case["format"]
    if case["op"] == "cache":
        n = case["rows"]
        n_pages = int(math.ceil(case["spare"] * n / page)) + 1
        # rows differ in size as heads and tokens do
        st["k"] = (normal(n, hkv, dh) * (2.0 * normal(n, hkv, 1)).exp2()).to(dtype)
        st["v"] = (normal(n, hkv, dh) * (2.0 * normal(n, hkv, 1)).exp2()).to(dtype)
        st["k_out"], st["v_out"] = torch.empty_like(st["k"]), torch.empty_like(st["v"])
        if n <= 256:            # tokens of as many sequences: anywhere
            slots = torch.randperm(n_pages * page, generator=g, device="cuda")[:n]
        else:                   # one sequence: whole pages in any order
            order = torch.randperm(n_pages, generator=g, device="cuda")
            slots = (order[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:n]
        st["slots"] = slots.to(torch.int32)
    else:
        new, total = _lens(case)
        per = [-(-t // page) for t in total]
        n_pages, width = sum(per) + 3, max(per)
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros((case["seqs"], width), dtype=torch.int32, device="cuda")
        at = 0
        for s, p in enumerate(per):
            table[s, :p] = order[at:at + p]
            at += p
        st["table"], st["new"], st["total"] = table, new, total
        st["kv_len"] = torch.tensor(total, dtype=torch.int32, device="cuda")
        st["q_start"] = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
        rows = sum(new)
        st["q"] = normal(rows, hq, dh).to(dtype)
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((rows, hq), dtype=torch.float32, device="cuda")
    shape = (n_pages, hkv, page, dh)
    for x in ("k", "v"):
        if fmt in LIMIT:
            st[x + "_scale"] = torch.zeros(shape[:3], device="cuda")
        if case["op"] == "cache":
            st[x + "_pages"] = torch.zeros(shape, dtype=TYPES[fmt], device="cuda")
            continue
        st[x + "_pages"] = torch.empty(shape, dtype=TYPES[fmt], device="cuda")
        step = max(1, (1 << 26) // (hkv * page * dh))
        for p in range(0, n_pages, step):
            part = normal(min(step, n_pages - p), *shape[1:])
            if fmt in LIMIT:
                codes, st[x + "_scale"][p:p + step] = _quantise(part, fmt)
                st[x + "_pages"][p:p + step] = codes
            else:
                st[x + "_pages"][p:p + step] = part.to(TYPES[fmt])
    if own:
        _own_cache(st)
    return st


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        return {"rope": _own_rope, "cache": _own_write_read, "attend": _own_attend, "sample": _own_sample}[op](state)
    return {"rope": _plain_rope, "cache": _plain_write_read, "attend": _plain_attend, "sample": _plain_sample}[op](state)


def _own_rope(st):
    from paper_2602_23592_amd import binding as kb
    c = st["case"]
    kb.rope_rows(st["q"], st["k"], st["positions"], st["freq"],
                 layout=kb.KEEP_ROPE_HALF if c["layout"] == "half" else kb.KEEP_ROPE_INTERLEAVED,
                 magnitude=st["magnitude"], q_out=st["q_out"], k_out=st["k_out"])
    return {"q": st["q_out"], "k": st["k_out"]}


def _own_cache(st):
    """The handle of the pages and, for attention, its workspace: made once, as a serving program does."""
    from paper_2602_23592_amd import binding as kb
    if "handle" not in st:
        st["handle"] = kb.PagedCache(st["k_pages"], st["v_pages"], st.get("k_scale"), st.get("v_scale"))
        if st["case"]["op"] == "attend":
            hq, _, dh = HEADS[st["case"]["heads"]]
            st["workspace"] = torch.empty(kb.paged_attention_workspace_bytes(hq, st["handle"], st["case"]["seqs"]),
                                          dtype=torch.uint8, device="cuda")
    return st["handle"]


def _own_write_read(st):
    h = _own_cache(st)
    h.write(st["k"], st["v"], st["slots"])
    h.read(st["slots"], st["k_out"], st["v_out"])
    return {"k": st["k_out"], "v": st["v_out"]}


def _own_attend(st):
    from paper_2602_23592_amd import binding as kb
    h = _own_cache(st)
    kb.paged_attention(st["q"], h, st["q_start"], st["kv_len"], st["table"], window=st["case"]["window"], out=st["out"],
                       lse=st["lse"], workspace=st["workspace"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_sample_workspace(st):
    from paper_2602_23592_amd import binding as kb
    if "workspace" not in st:
        st["workspace"] = torch.empty(kb.sample_workspace_bytes(st["case"]["rows"], st["case"]["vocab"]), dtype=torch.uint8,
                                      device="cuda")
    return st["workspace"]


def _own_sample(st):
    from paper_2602_23592_amd import binding as kb
    kb.sample(st["logits"], st["uniform"], st["temperature"], st["top_k"], st["top_p"], st["min_p"], tokens=st["tokens"],
              probs=st["probs"], workspace=_own_sample_workspace(st))
    return {"tokens": st["tokens"], "probs": st["probs"]}


def _plain_rope(st):
    c = st["case"]
    rot = c["rot"]
    a = st["positions"].double()[:, None, None] * st["freq"]
    cos, sin = (a.cos() * st["magnitude"]).float(), (a.sin() * st["magnitude"]).float()
    res = {}
    for x in ("q", "k"):
        t = st[x].float()
        y = t.clone()
        if c["layout"] == "half":
            x1, x2 = t[..., :rot // 2], t[..., rot // 2:rot]
            y[..., :rot // 2], y[..., rot // 2:rot] = x1 * cos - x2 * sin, x2 * cos + x1 * sin
        else:
            x1, x2 = t[..., 0:rot:2], t[..., 1:rot:2]
            y[..., 0:rot:2], y[..., 1:rot:2] = x1 * cos - x2 * sin, x2 * cos + x1 * sin
        res[x] = y.to(st[x].dtype)
    return res


def _quantise(x, fmt):
    """codes and scales of fp32 rows: the largest magnitude becomes the largest code"""
    top = LIMIT[fmt]
    scale = (x.abs().amax(-1) / top).clamp(min=2.0 ** -126)
    y = (x / scale[..., None]).clamp(-top, top)
    return (y.round() if fmt == "int8" else y).to(TYPES[fmt]), scale


def _plain_write_read(st):
    c = st["case"]
    page, fmt = c["page"], c["format"]
    at = st["slots"].long()
    p, o = at // page, at % page
    res = {}
    for x in ("k", "v"):
        pages, t = st[x + "_pages"], st[x].float()
        if fmt in LIMIT:
            codes, scale = _quantise(t, fmt)
            pages.view(torch.uint8)[p, :, o] = codes.view(torch.uint8)
            st[x + "_scale"][p, :, o] = scale
            back = pages.view(torch.uint8)[p, :, o].view(pages.dtype).float() * st[x + "_scale"][p, :, o][..., None]
        else:
            pages[p, :, o] = t.to(pages.dtype)
            back = pages[p, :, o].float()
        res[x] = back.to(st[x].dtype)
    return res


def _keys(st, x, s, f):
    """keys or values of sequence s, [tokens, heads, dh], as type f"""
    n = st["total"][s]
    pages = st["table"][s, :-(-n // st["case"]["page"])].long()
    t = st[x + "_pages"]
    t = t.view(torch.uint8)[pages].view(t.dtype).to(f) if t.dtype == torch.float8_e4m3fn else t[pages].to(f)
    if x + "_scale" in st:
        t = t * st[x + "_scale"][pages].to(f)[..., None]
    return t.permute(0, 2, 1, 3).flatten(0, 1)[:n]


def _plain_attend(st):
    c = st["case"]
    hq, hkv, dh = HEADS[c["heads"]]
    rep, w = hq // hkv, c["window"] or 1 << 30
    out = torch.empty_like(st["q"])
    lse = torch.empty_like(st["lse"])
    row = 0
    for s, (n, total) in enumerate(zip(st["new"], st["total"])):
        k = _keys(st, "k", s, torch.float32).permute(1, 2, 0).contiguous()       # [hkv, dh, keys]
        v = _keys(st, "v", s, torch.float32).permute(1, 0, 2).contiguous()
        key = torch.arange(total, device="cuda")
        step = max(1, (1 << 28) // (hq * total))
        for i in range(0, n, step):
            m = min(step, n - i)
            q = st["q"][row + i:row + i + m].float().view(m, hkv, rep, dh).permute(1, 2, 0, 3).reshape(hkv, rep * m, dh)
            x = (torch.bmm(q, k) / math.sqrt(dh)).view(hkv, rep, m, total)
            pos = (total - n + i + torch.arange(m, device="cuda"))[:, None]
            x = x.masked_fill((key > pos) | (key <= pos - w), -math.inf)
            top = x.amax(-1, keepdim=True)
            x = (x - top).exp_()
            den = x.sum(-1, keepdim=True)
            o = torch.bmm(x.view(hkv, rep * m, total), v).view(hkv, rep, m, dh) / den
            out[row + i:row + i + m] = o.permute(2, 0, 1, 3).reshape(m, hq, dh).to(out.dtype)
            lse[row + i:row + i + m] = (top + den.log())[..., 0].permute(2, 0, 1).reshape(m, hq)
        row += n
    return {"out": out, "lse": lse}


def _plain_sample(st):
    tokens, probs = [], []
    step = max(1, (1 << 25) // st["case"]["vocab"])
    for i in range(0, st["case"]["rows"], step):
        x = st["logits"][i:i + step].double()
        t = st["temperature"][i:i + step, None].double()
        x, order = x.sort(dim=-1, descending=True, stable=True)
        greedy = t <= 0
        w = ((x - x[:, :1]) / torch.where(greedy, 1.0, t)).exp_().mul_(WEIGHT_ONE).round_().to(torch.int64)
        w[:, 1:] *= (~greedy).long()
        # a token stays if it weighs at least min_p of the likeliest, ranks among the top_k and starts below top_p of them
        w *= w >= (st["min_p"][i:i + step, None].double() * WEIGHT_ONE).ceil().long()
        k = st["top_k"][i:i + step, None]
        w *= (k <= 0) | (torch.arange(w.shape[1], device="cuda") < k)
        cum = w.cumsum(-1)
        keep = (st["top_p"][i:i + step, None].double() * cum[:, -1:].double()).ceil().long().clamp(min=1)
        w *= cum - w < keep
        total = w.sum(-1, keepdim=True)
        goal = torch.minimum((st["uniform"][i:i + step, None].double() * total.double()).floor().long(), total - 1)
        at = (cum <= goal).sum(-1, keepdim=True)
        tokens.append(order.gather(-1, at)[:, 0].to(torch.int32))
        probs.append((w.gather(-1, at).double() / total.double())[:, 0].float())
    return {"tokens": torch.cat(tokens), "probs": torch.cat(probs)}


# ---------------------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] == "sample" and case["rows"] * case["vocab"] > 1 << 27:
        return None
    if case["op"] == "attend" and 2 * _pairs(case)[0] * HEADS[case["heads"]][0] * HEADS[case["heads"]][2] > 4e12:
        return None
    st = prepare(case, seed)
    return {"rope": _exact_rope, "cache": _exact_cache, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](st)


def _exact_rope(st):
    """Pairs as complex numbers, turned by multiplication."""
    c = st["case"]
    rot = c["rot"]
    turn = torch.polar(torch.full((), st["magnitude"], dtype=torch.float64, device="cuda").expand(c["rows"], rot // 2),
                       torch.outer(st["positions"].double(), st["freq"]))
    res = {}
    for x in ("q", "k"):
        y = st[x].double()
        head = y[..., :rot]
        pairs = head.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if c["layout"] == "half" else head.unflatten(-1, (rot // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        y[..., :rot] = (z.transpose(-1, -2) if c["layout"] == "half" else z).flatten(-2)
        res[x] = y
    return res


def _exact_cache(st):
    """The stored value nearest to each element, by the format's own grid; the scales are fp32 by definition."""
    fmt = st["case"]["format"]
    res = {}
    for x in ("k", "v"):
        t = st[x].double()
        if fmt not in LIMIT:
            res[x] = st[x].to(TYPES[fmt]).double()
            continue
        scale = torch.clamp(st[x].float().abs().amax(-1) / LIMIT[fmt], min=2.0 ** -126)[..., None]
        u = torch.clamp((st[x].float() / scale).double(), -LIMIT[fmt], LIMIT[fmt])
        if fmt == "int8":
            grid = torch.ones_like(u)
        else:                   # four bits of significand; below 2^-6 a fixed step of 2^-9
            grid = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
        res[x] = torch.round(u / grid) * grid * scale.double()
    return res


def _exact_attend(st):
    c = st["case"]
    hq, hkv, dh = HEADS[c["heads"]]
    rep, w = hq // hkv, c["window"] or 1 << 30
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for s, (n, total) in enumerate(zip(st["new"], st["total"])):
        ks, vs = _keys(st, "k", s, torch.float64), _keys(st, "v", s, torch.float64)
        first = total - n - torch.arange(total, device="cuda")           # distance of row 0 from each key
        step = max(1, (1 << 27) // total)
        for h in range(hq):
            kt, vt = ks[:, h // rep].t().contiguous(), vs[:, h // rep].contiguous()
            for i in range(0, n, step):
                a, b = row + i, row + min(n, i + step)
                x = torch.mm(st["q"][a:b, h].double(), kt) * dh ** -0.5
                d = first[None] + torch.arange(i, min(n, i + step), device="cuda")[:, None]
                x.masked_fill_((d < 0) | (d >= w), -math.inf)
                lse[a:b, h] = x.logsumexp(-1)
                out[a:b, h] = torch.mm((x - lse[a:b, h, None]).exp_(), vt)
        row += n
    return {"out": out, "lse": lse}


def _exact_sample(st):
    """Row by row on the host, with Python's whole numbers for the sums that decide."""
    x = st["logits"].double().cpu().numpy()
    par = {n: st[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p", "uniform")}
    tokens, probs = np.zeros(len(x), np.int32), np.zeros(len(x))
    for r, row in enumerate(x):
        t = par["temperature"][r]
        best = int(np.argmax(row))
        tokens[r], probs[r] = best, 1.0
        if t <= 0:
            continue
        w = np.rint(np.exp((row - row[best]) / t) * WEIGHT_ONE)
        ids = np.flatnonzero((w >= max(1.0, math.ceil(par["min_p"][r] * WEIGHT_ONE))))
        ids = ids[np.lexsort((ids, -row[ids]))]
        if par["top_k"][r] > 0:
            ids = ids[:int(par["top_k"][r])]
        wi = w[ids].astype(np.int64)
        ends = np.cumsum(wi)
        goal = max(1, math.ceil(par["top_p"][r] * float(int(ends[-1]))))
        n = int(np.searchsorted(ends, goal, side="left")) + 1
        n = min(n, len(ids))
        total = int(ends[n - 1])
        at = int(np.searchsorted(ends[:n], min(total - 1, math.floor(par["uniform"][r] * float(total))), side="right"))
        tokens[r], probs[r] = ids[at], int(wi[at]) / total
    return {"tokens": tokens, "probs": probs}
