"""The work of a token decoder behind a CNN trunk, as cases that can be timed
and checked: attention over packed prompts, the paged cache that holds keys
and values in 4 bits (writing and reading it, moving its pages), and single
token attention over that cache.

A convolutional trunk hands its feature maps over as tokens: the 8x8, 28x28,
35x35, 42x42 and 55x55 maps of this repository's blocks are prompts of 64, 784,
1225, 1764 and 3025 tokens.  A decoder attends over them once, keeps their keys
and values, and then answers one token at a time, for several answers of one
image at once (forked sequences that share their prompt's pages).

``run`` computes an operator in elementary torch operations in 32 bits where
``own`` is false, and through the library's entry points where it is true.

The 4-bit format, for 32 consecutive values x of one head's key or value (all
steps in float32, each rounded once):

    x   = min(max(x, -61440), 61440)          (so that z + s c stays within f16)
    z   = f16(min x),  s = f16((max x - min x) * f32(1 / 15))
    c_i = min(max(round_half_even((x_i - z) / s), 0), 15), 0 where s = 0
    the value that is held: z + s c_i
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
GROUP = 32                       # values that share a scale and a zero point
LIMIT = 61440.0


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one 8x8 map, one request: launch latency
        {"name": "prompt_8x8", "op": "prompt", "dtype": "bf16", "heads": 8, "kv_heads": 2, "head_dim": 64,
         "lens_q": "64", "lens_k": "64", "causal": True},
        # feature maps of several trunks packed behind each other, among them the last part of a map whose first
        # part is already there, and a single token
        {"name": "prompt_maps", "op": "prompt", "dtype": "f16", "heads": 16, "kv_heads": 4, "head_dim": 64,
         "lens_q": "784,1225,512,49,1,3025", "lens_k": "784,1225,1764,49,900,3025", "causal": True},
        # float32, the trunk's own type, as many heads of keys as of queries, every token seeing its whole map
        {"name": "prompt_float", "op": "prompt", "dtype": "f32", "heads": 12, "kv_heads": 12, "head_dim": 96,
         "lens_q": "1225,784,193", "lens_k": "1225,784,193", "causal": False},
        # one long prompt: the rate of the matrix cores
        {"name": "prompt_long", "op": "prompt", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "lens_q": "16384", "lens_k": "16384", "causal": True},
        # one token after one 28x28 map: launch latency
        {"name": "decode_28x28", "op": "decode", "dtype": "f16", "heads": 8, "kv_heads": 2, "head_dim": 64,
         "page": 32, "lens": "785"},
        # a batch of answers over maps of every size, ragged
        {"name": "decode_maps", "op": "decode", "dtype": "bf16", "heads": 16, "kv_heads": 4, "head_dim": 96,
         "page": 32, "lens": "65,785,1226,1765,3026,1,33,129,801,1240,1799,3100,97,790,1300,2048"},
        # one sequence with a long cache and few rows: the work has to be split along the cache
        {"name": "decode_one_long", "op": "decode", "dtype": "bf16", "heads": 16, "kv_heads": 2, "head_dim": 128,
         "page": 128, "lens": "131072"},
        # a full batch of long sequences: the rate of the memory
        {"name": "decode_batch", "op": "decode", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "lens": ",".join(str(8192 + 769 * i) for i in range(32))},
        # the newest token of every sequence of a batch, written to the cache and read back
        {"name": "write_tokens", "op": "write", "dtype": "bf16", "kv_heads": 8, "head_dim": 128, "page": 64,
         "lens": ",".join(str(64 + 97 * i) for i in range(32)), "new": ",".join(["1"] * 32)},
        # whole prompts written to the cache and read back
        {"name": "write_prompts", "op": "write", "dtype": "bf16", "kv_heads": 8, "head_dim": 128, "page": 64,
         "lens": "3025,1764,16384,1225,784,12289", "new": "3025,1764,16384,1225,784,12289"},
        # four images, four answers each: fork, and room for the first new token of every answer
        {"name": "pages_fork", "op": "fork", "layers": 4, "kv_heads": 2, "head_dim": 64, "page": 32, "pages": 512,
         "lens": "785,1226,1760,3025", "children": 4},
        # a pool from which a third of the sequences has gone: what is left moves to the front
        {"name": "pages_compact", "op": "compact", "layers": 8, "kv_heads": 8, "head_dim": 128, "page": 64,
         "pages": 512, "slots": 24, "len": 1225},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["prompt", "prompt", "decode", "decode", "write", "fork", "compact"])
    kv = rng.choice([1, 2, 3, 4, 8])
    page = rng.choice([32, 64, 128, 256])
    dtype = rng.choice(["f16", "bf16"])
    dim = rng.choice([32, 64, 96, 128])
    if op == "prompt":
        dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
        n = rng.randint(1, 6)
        lens_k = [_log(rng, 1, 2000 if dtype == "f32" else 6000) for _ in range(n)]
        lens_q = [m if rng.random() < 0.7 else _log(rng, 1, m) for m in lens_k]
        return {"op": op, "dtype": dtype, "heads": kv * rng.choice([1, 2, 4, 6, 8]) if kv < 8 else 32, "kv_heads": kv,
                "head_dim": rng.choice([32, 40, 64, 80, 96, 128]), "lens_q": ",".join(map(str, lens_q)),
                "lens_k": ",".join(map(str, lens_k)), "causal": rng.random() < 0.8}
    if op == "decode":
        lens = [_log(rng, 1, 40000) for _ in range(_log(rng, 1, 32))]
        return {"op": op, "dtype": dtype, "heads": kv * rng.choice([1, 2, 4, 5, 8]), "kv_heads": kv, "head_dim": dim,
                "page": page, "lens": ",".join(map(str, lens))}
    if op == "write":
        lens = [_log(rng, 1, 8000) for _ in range(_log(rng, 1, 16))]
        new = [1] * len(lens) if rng.random() < 0.4 else [_log(rng, 1, m) for m in lens]
        return {"op": op, "dtype": rng.choice(["f16", "bf16", "f32"]), "kv_heads": kv, "head_dim": dim, "page": page,
                "lens": ",".join(map(str, lens)), "new": ",".join(map(str, new))}
    layers = _log(rng, 1, 8)
    if op == "fork":
        lens = [_log(rng, 1, 4000) for _ in range(rng.randint(1, 6))]
        children = rng.randint(1, 6)
        need = sum(_pages(m, page) for m in lens) + len(lens) * children
        return {"op": op, "layers": layers, "kv_heads": kv, "head_dim": dim, "page": page,
                "pages": need + rng.randint(0, 64), "lens": ",".join(map(str, lens)), "children": children}
    slots, length = rng.randint(3, 30), _log(rng, 10, 7 * page)
    return {"op": op, "layers": layers, "kv_heads": kv, "head_dim": dim, "page": page,
            "pages": slots * _pages(length, page) + rng.randint(1, 40), "slots": slots, "len": length}


def _ints(text):
    return [int(v) for v in text.split(",")]


def _pages(tokens, page):
    return -(-tokens // page)


def _page_bytes(case):
    """Bytes of a page in one layer: codes, and a scale and a zero point in f16 for every 32 of them."""
    return case["kv_heads"] * case["page"] * 2 * (case["head_dim"] // 2 + 4 * case["head_dim"] // GROUP)


def _pairs(lq, lk, causal):
    """Pairs of a query and a key that it sees: the last query sees every key."""
    if not causal:
        return lq * lk
    return sum(max(0, lk - lq + i + 1) for i in range(lq))


def work(case):
    op = case["op"]
    if op == "prompt":
        lq, lk = _ints(case["lens_q"]), _ints(case["lens_k"])
        size = 4 if case["dtype"] == "f32" else 2
        d, h, kv = case["head_dim"], case["heads"], case["kv_heads"]
        return {"bytes": size * d * (2 * h * sum(lq) + 2 * kv * sum(lk)),
                "flops": 4 * d * h * sum(_pairs(a, b, case["causal"]) for a, b in zip(lq, lk))}
    if op == "decode":
        lens = _ints(case["lens"])
        d, h, kv = case["head_dim"], case["heads"], case["kv_heads"]
        return {"bytes": sum(lens) * kv * 2 * (d // 2 + 4 * d // GROUP) + 2 * 2 * len(lens) * h * d,
                "flops": 4 * d * h * sum(lens)}
    if op == "write":     # the input, the cache written and read, the values in 32 bits
        values = 2 * sum(_ints(case["new"])) * case["kv_heads"] * case["head_dim"]
        return {"bytes": values * (4 if case["dtype"] == "f32" else 2) + 2 * values * 5 // 8 + 4 * values,
                "flops": 8 * values}
    if op == "fork":
        lens = _ints(case["lens"])
        copies = case["children"] * sum(1 for m in lens if m % case["page"])
        entries = case["children"] * sum(_pages(m, case["page"]) for m in lens)
        return {"bytes": 2 * copies * case["layers"] * _page_bytes(case) + 3 * 8 * entries + 4 * case["pages"],
                "flops": 0}
    table, refs, _ = _fragmented(case)
    live = sum(1 for r in refs if r)
    moved = sum(1 for p, r in enumerate(refs) if r and p >= live)
    return {"bytes": 2 * moved * case["layers"] * _page_bytes(case) + 8 * len(refs) + 8 * len(table) * len(table[0]),
            "flops": 0}


def _fragmented(case):
    """Sequences that grew page by page in turn; every third has been freed,
    and the one after it shares its first half with the one before."""
    slots, page = case["slots"], case["page"]
    row = _pages(case["len"], page) + 1
    lens = [max(1, case["len"] * (slots + i) // (2 * slots)) for i in range(slots)]
    table = [[-1] * row for _ in range(slots)]
    refs = [0] * case["pages"]
    at = 0
    for j in range(row):
        for i in range(slots):
            if j < _pages(lens[i], page):
                table[i][j] = at
                refs[at] = 1
                at += 1
    for i in range(1, slots, 3):
        for j in range(row):
            if table[i][j] >= 0:
                refs[table[i][j]] -= 1
        table[i], lens[i] = [-1] * row, 0
        if i + 1 < slots:
            for j in range(_pages(lens[i - 1], page) // 2):
                refs[table[i + 1][j]] -= 1
                table[i + 1][j] = table[i - 1][j]
                refs[table[i - 1][j]] += 1
    return table, refs, lens


# ---------------------------------------------------------------- inputs

def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _offsets(lens):
    out = [0]
    for m in lens:
        out.append(out[-1] + m)
    return out


def _rng(seed, part):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + part)


def _kv(case, tokens, seed, part):
    """Keys and values as one projection leaves them, [tokens][2][kv_heads][head_dim]: some key channels are
    much larger than the others, the values' heads differ in size."""
    g, kv, d = _rng(seed, part), case["kv_heads"], case["head_dim"]
    x = torch.randn(tokens, 2, kv, d, generator=g, device=DEV)
    channel = torch.randn(kv, d, generator=_rng(seed, 1), device=DEV)
    x[:, 0] = x[:, 0] * torch.exp(0.5 * channel) + 0.5 * channel
    x[:, 1] *= torch.exp(torch.randn(kv, 1, generator=_rng(seed, 2), device=DEV))
    return x.to(DTYPES[case["dtype"]])


def _queries(case, tokens, seed):
    x = torch.randn(tokens, case["heads"], case["head_dim"], generator=_rng(seed, 0), device=DEV)
    return x.to(DTYPES[case["dtype"]])


def _shuffled_table(case, lens, seed):
    """Pages of sequences that grew side by side: in no order."""
    counts = [_pages(m, case["page"]) for m in lens]
    order = list(range(sum(counts)))
    random.Random(seed).shuffle(order)
    table, at = [], 0
    for c in counts:
        table.append(order[at:at + c] + [-1] * (max(counts) - c))
        at += c
    return table, [1] * len(order)


def _cache(case, layers, table, refs, lens, pool=None):
    """The library's description of a cache, and the tensors that it points to."""
    import paper_2011_01302_amd as I
    st = {"refs": _i32(refs), "table": _i32(table), "lens": _i32(lens)}
    c = I.ios_cache()
    c.layers, c.kv_heads, c.head_dim, c.page_tokens = layers, case["kv_heads"], case["head_dim"], case["page"]
    c.pages, c.slots, c.row = len(refs), len(table), len(table[0])
    st["pool"] = pool if pool is not None else torch.zeros(layers, len(refs), I.ios_cache_page_bytes(c),
                                                           dtype=torch.uint8, device=DEV)
    st["work"] = torch.zeros(I.ios_cache_work_bytes(c), dtype=torch.uint8, device=DEV)
    c.pool, c.refs, c.table, c.lens = (st[n].data_ptr() for n in ("pool", "refs", "table", "lens"))
    c.work = st["work"].data_ptr()
    st["cache"] = c
    return st


def _tokens(t):
    """[tokens][heads][head_dim], the last dimension contiguous."""
    import paper_2011_01302_amd as I
    return I.ios_tokens(t.data_ptr(), t.shape[0], t.stride(0), t.stride(1))


def _attn_desc(case, seqs, max_keys):
    import paper_2011_01302_amd as I
    d = I.ios_attn_desc()
    d.dtype = {"f32": I.IOS_F32, "f16": I.IOS_F16, "bf16": I.IOS_BF16}[case["dtype"]]
    d.heads, d.kv_heads, d.head_dim = case["heads"], case["kv_heads"], case["head_dim"]
    d.seqs, d.max_keys, d.scale = seqs, max_keys, 1.0 / math.sqrt(case["head_dim"])
    d.causal = 1 if case.get("causal") else 0
    return d


def prepare(case, seed):
    st = {"case": case}
    op = case["op"]
    if op == "prompt":
        lq, lk = _ints(case["lens_q"]), _ints(case["lens_k"])
        st["lens_q"], st["lens_k"] = lq, lk
        st["cu_q"], st["cu_k"] = _i32(_offsets(lq)), _i32(_offsets(lk))
        st["q"] = _queries(case, sum(lq), seed)
        kv = _kv(case, sum(lk), seed, 3)
        st["k"], st["v"] = kv[:, 0], kv[:, 1]
        if own:
            import paper_2011_01302_amd as I
            st["desc"] = _attn_desc(case, len(lq), max(lk))
            n = I.ios_attn_work_bytes(st["desc"], sum(lq))
            st["work"], st["work_bytes"] = torch.zeros(max(n, 1), dtype=torch.uint8, device=DEV), n
    elif op == "decode":
        lens = _ints(case["lens"])
        st["q"] = _queries(case, len(lens), seed)
        if own:
            import paper_2011_01302_amd as I
            st.update(_cache(case, 1, *_shuffled_table(case, lens, seed), lens))
            st["desc"] = _attn_desc(case, len(lens), max(lens))
            n = I.ios_attn_work_bytes(st["desc"], len(lens))
            st["attn_work"], st["work_bytes"] = torch.zeros(max(n, 1), dtype=torch.uint8, device=DEV), n
            st["seqs"] = _i32(list(range(len(lens))))
        st["held"] = []
        for i, m in enumerate(lens):
            kv = _kv(case, m, seed, 3 + i)
            if own:
                cu = _i32([0, m])
                I.ios_cache_append(st["cache"], 0, st["desc"].dtype, _tokens(kv[:, 0]), _tokens(kv[:, 1]), 1,
                                   st["seqs"][i:].data_ptr(), cu.data_ptr(), _stream())
            else:
                st["held"].append((_quantised(kv[:, 0]), _quantised(kv[:, 1])))
    elif op == "write":
        lens, new = _ints(case["lens"]), _ints(case["new"])
        kv = _kv(case, sum(new), seed, 3)
        st["k"], st["v"] = kv[:, 0], kv[:, 1]
        if own:
            st.update(_cache(case, 1, *_shuffled_table(case, lens, seed), lens))
            st["seqs"], st["cu"] = _i32(list(range(len(lens)))), _i32(_offsets(new))
    else:
        if op == "fork":
            parents = _ints(case["lens"])
            n, lens = len(parents), parents + [0] * (len(parents) * case["children"])
            row = max(_pages(m, case["page"]) for m in parents) + 1
            table, at = [], 0
            for m in lens:
                c = _pages(m, case["page"])
                table.append(list(range(at, at + c)) + [-1] * (row - c))
                at += c
            refs = [1] * at + [0] * (case["pages"] - at)
            pairs = [(p, n + p * case["children"] + j) for p in range(n) for j in range(case["children"])]
            st["parents"], st["children"] = _i32([p for p, _ in pairs]), _i32([c for _, c in pairs])
            st["add"] = _i32([1] * len(pairs))
        else:
            table, refs, lens = _fragmented(case)
            st["table0"], st["refs0"] = _i32(table), _i32(refs)
            st["live"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        pool = torch.randint(0, 256, (case["layers"], len(refs), _page_bytes(case)), dtype=torch.uint8, device=DEV,
                             generator=_rng(seed, 0))
        if own:
            st.update(_cache(case, case["layers"], table, refs, lens, pool))
        else:
            st.update(pool=pool, table=_i32(table), refs=_i32(refs), lens=_i32(lens))
    return st


# ---------------------------------------------------------------- one pass

def _stream():
    return torch.cuda.current_stream().cuda_stream


def run(st):
    op = st["case"]["op"]
    if own:
        return {"prompt": _own_prompt, "decode": _own_decode, "write": _own_write, "fork": _own_fork,
                "compact": _own_compact}[op](st)
    return {"prompt": _plain_prompt, "decode": _plain_decode, "write": _plain_write, "fork": _plain_fork,
            "compact": _plain_compact}[op](st)


def _own_prompt(st):
    import paper_2011_01302_amd as I
    out = torch.empty_like(st["q"])
    I.ios_attn_prompt(st["desc"], _tokens(st["q"]), _tokens(st["k"]), _tokens(st["v"]), _tokens(out), 0,
                      st["cu_q"].data_ptr(), st["cu_k"].data_ptr(), st["work"].data_ptr(), st["work_bytes"], _stream())
    return out


def _own_decode(st):
    import paper_2011_01302_amd as I
    out = torch.empty_like(st["q"])
    I.ios_attn_cache(st["cache"], 0, st["desc"], _tokens(st["q"]), _tokens(out), 0, st["seqs"].data_ptr(),
                     st["attn_work"].data_ptr(), st["work_bytes"], _stream())
    return out


def _own_write(st):
    import paper_2011_01302_amd as I
    k, v, n, s = st["k"], st["v"], st["seqs"].shape[0], _stream()
    dtype = {torch.float32: I.IOS_F32, torch.float16: I.IOS_F16, torch.bfloat16: I.IOS_BF16}[k.dtype]
    ko = torch.empty(k.shape, dtype=torch.float32, device=DEV)
    vo = torch.empty_like(ko)
    I.ios_cache_append(st["cache"], 0, dtype, _tokens(k), _tokens(v), n, st["seqs"].data_ptr(), st["cu"].data_ptr(), s)
    I.ios_cache_read(st["cache"], 0, I.IOS_F32, _tokens(ko), _tokens(vo), n, st["seqs"].data_ptr(),
                     st["cu"].data_ptr(), s)
    return ko, vo


def _own_fork(st):
    import paper_2011_01302_amd as I
    c, n, s = st["cache"], st["children"].shape[0], _stream()
    I.ios_cache_free(c, n, st["children"].data_ptr(), s)          # the answers of the pass before
    I.ios_cache_fork(c, n, st["parents"].data_ptr(), st["children"].data_ptr(), s)
    I.ios_cache_reserve(c, n, st["children"].data_ptr(), st["add"].data_ptr(), s)
    return {"pool": st["pool"], "table": st["table"], "refs": st["refs"], "lens": st["lens"]}


def _own_compact(st):
    import paper_2011_01302_amd as I
    st["table"].copy_(st["table0"])        # as the sequences that are gone left it
    st["refs"].copy_(st["refs0"])
    I.ios_cache_compact(st["cache"], st["live"].data_ptr(), _stream())
    return {"pool": st["pool"], "table": st["table"], "refs": st["refs"], "live": st["live"]}


def _plain_prompt(st):
    q, k, v = st["q"], st["k"], st["v"]
    h, kv, d = q.shape[1], k.shape[1], q.shape[2]
    scale = 1.0 / math.sqrt(d)
    out = torch.empty_like(q)
    aq = ak = 0
    for lq, lk in zip(st["lens_q"], st["lens_k"]):
        for g in range(kv):
            heads = slice(g * (h // kv), (g + 1) * (h // kv))
            kk = k[ak:ak + lk, g].float()
            vv = v[ak:ak + lk, g].float()
            for i in range(0, lq, 4096):           # parts of the queries, so that the scores fit
                qq = q[aq + i:aq + min(i + 4096, lq), heads].float().transpose(0, 1)
                s = torch.matmul(qq, kk.t()) * scale
                if st["case"]["causal"]:
                    row = torch.arange(i, i + qq.shape[1], device=DEV)[:, None] + (lk - lq)
                    s.masked_fill_(torch.arange(lk, device=DEV)[None] > row, float("-inf"))
                p = torch.exp(s - s.amax(-1, keepdim=True))
                o = torch.matmul(p, vv) / p.sum(-1, keepdim=True)
                out[aq + i:aq + i + qq.shape[1], heads] = o.transpose(0, 1).to(q.dtype)
        aq, ak = aq + lq, ak + lk
    return out


def _quantised(x):
    """Codes, scales and zero points of x [tokens][heads][head_dim]."""
    x = x.float().clamp(-LIMIT, LIMIT).unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    z = lo.half()
    s = ((hi - lo) * torch.tensor(1.0 / 15.0, device=x.device)).half()
    c = torch.where(s > 0, torch.round((x - z.float()) / s.float()).clamp(0, 15), 0.0)
    return c.to(torch.uint8), s, z


def _values(held):
    c, s, z = held
    return (z.float() + s.float() * c.float()).flatten(-2)


def _plain_decode(st):
    q = st["q"]
    out = torch.empty_like(q)
    for i, (hk, hv) in enumerate(st["held"]):
        k, v = _values(hk).transpose(0, 1), _values(hv).transpose(0, 1)      # [kv_heads][tokens][head_dim]
        qq = q[i].float().unflatten(0, (k.shape[0], -1))
        s = torch.matmul(qq, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(q.shape[-1]))
        p = torch.exp(s - s.amax(-1, keepdim=True))
        out[i] = (torch.matmul(p, v.contiguous()) / p.sum(-1, keepdim=True)).flatten(0, 1).to(q.dtype)
    return out


def _plain_write(st):
    return _values(_quantised(st["k"])), _values(_quantised(st["v"]))


def _plain_free(st, slots):
    pages = st["table"][slots.long()].flatten()
    pages = pages[pages >= 0].long()
    st["refs"].index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))
    st["table"][slots.long()] = -1
    st["lens"][slots.long()] = 0


def _plain_fork(st):
    table, refs, lens, pool = st["table"], st["refs"], st["lens"], st["pool"]
    kids, page = st["children"].long(), st["case"]["page"]
    _plain_free(st, kids)
    table[kids] = table[st["parents"].long()]
    lens[kids] = lens[st["parents"].long()]
    pages = table[kids].flatten()
    pages = pages[pages >= 0].long()
    refs.index_add_(0, pages, torch.ones_like(pages, dtype=torch.int32))
    # room for one token more: a page of its own in the place of a shared last page, or a new page
    at = lens[kids].long()
    last = table[kids, torch.clamp((at - 1) // page, min=0)].long()
    shared = at % page != 0
    grow = (at % page == 0)
    free = torch.nonzero(refs == 0).flatten()
    need = (shared | grow).long()
    mine = free[torch.cumsum(need, 0) - need]
    src, dst = last[shared], mine[shared]
    pool[:, dst] = pool[:, src]
    refs.index_add_(0, src, torch.full_like(src, -1, dtype=torch.int32))
    table[kids, at // page] = mine.to(torch.int32)
    refs[mine] = 1
    lens[kids] += st["add"]
    return {"pool": pool, "table": table, "refs": refs, "lens": lens}


def _plain_compact(st):
    table, refs, pool = st["table"], st["refs"], st["pool"]
    table.copy_(st["table0"])
    refs.copy_(st["refs0"])
    held = refs > 0
    live = held.sum()
    at = torch.arange(refs.shape[0], device=DEV)
    src = torch.nonzero(held & (at >= live)).flatten()
    dst = torch.nonzero(~held & (at < live)).flatten()
    pool[:, dst] = pool[:, src]
    to = at.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].to(torch.int32), table))
    refs[dst] = refs[src]
    refs[src] = 0
    st["live"].copy_(live)
    return {"pool": pool, "table": table, "refs": refs, "live": st["live"]}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    op = case["op"]
    if op == "prompt":
        lens_q, lens_k = _ints(case["lens_q"]), _ints(case["lens_k"])
        q, kv = _queries(case, sum(lens_q), seed), _kv(case, sum(lens_k), seed, 3)
        out = torch.empty(q.shape, dtype=torch.float64, device=DEV)
        oq, ok = _offsets(lens_q), _offsets(lens_k)
        for i, (lq, lk) in enumerate(zip(lens_q, lens_k)):
            for h in range(case["heads"]):
                g = h * case["kv_heads"] // case["heads"]
                k, v = kv[ok[i]:ok[i] + lk, :, g].double().unbind(1)
                for a in range(0, lq, 2048):
                    b = min(lq, a + 2048)
                    seen = lk - lq + b if case["causal"] else lk      # later keys are seen by none of these
                    out[oq[i] + a:oq[i] + b, h] = _attend(q[oq[i] + a:oq[i] + b, h].double(), k[:seen], v[:seen],
                                                          lk - lq + a if case["causal"] else None)
        return out
    if op == "decode":
        q = _queries(case, len(_ints(case["lens"])), seed)
        out = torch.empty(q.shape, dtype=torch.float64, device=DEV)
        ratio = case["heads"] // case["kv_heads"]
        for i, m in enumerate(_ints(case["lens"])):
            kv = _held(_kv(case, m, seed, 3 + i))
            for g in range(case["kv_heads"]):
                rows = slice(g * ratio, (g + 1) * ratio)
                out[i, rows] = _attend(q[i, rows].double(), kv[:, 0, g], kv[:, 1, g], None)
        return out
    if op == "write":
        kv = _held(_kv(case, sum(_ints(case["new"])), seed, 3))
        return kv[:, 0], kv[:, 1]
    return _moved(case, seed)


def _attend(q, k, v, first):
    """Softmax attention of rows q; row r sees keys 0 .. first + r, or every key."""
    w = q @ k.T / math.sqrt(q.shape[1])
    if first is not None:
        hidden = torch.ones_like(w, dtype=torch.bool).triu(first + 1)
        w[hidden] = -math.inf
    w = (w - torch.logsumexp(w, 1, keepdim=True)).exp()
    return w @ v


def _held(x):
    """The values that the 4-bit format holds for x: its scale, zero point and codes are defined in 16 and 32
    bits, their sum is exact in 64."""
    y = torch.clip(x.to(torch.float32), -LIMIT, LIMIT).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    low, high = torch.aminmax(y, dim=-1, keepdim=True)
    zero, fifteenth = low.to(torch.float16).to(torch.float32), torch.full_like(low, 1.0 / 15.0)
    step = ((high - low) * fifteenth).to(torch.float16).to(torch.float32)
    code = torch.clip(torch.round(torch.nan_to_num((y - zero) / step, 0.0, 0.0, 0.0)), 0, 15)
    return (zero.double() + step.double() * code.double()).reshape(x.shape)


def _moved(case, seed):
    """Page by page on the host."""
    if case["op"] == "fork":
        parents, page, kids = _ints(case["lens"]), case["page"], case["children"]
        row = max(_pages(m, page) for m in parents) + 1
        table, lens, refs, copies, at = [], [], [0] * case["pages"], [], 0
        for m in parents:
            own_pages = list(range(at, at + _pages(m, page)))
            at += len(own_pages)
            table.append(own_pages)
            lens.append(m)
        for p, m in enumerate(parents):
            for _ in range(kids):
                rows = list(table[p])
                if m % page:
                    copies.append((rows.pop(), at))
                table.append(rows + [at])
                lens.append(m + 1)
                at += 1
        for rows in table:
            for p in rows:
                refs[p] += 1
        table = [rows + [-1] * (row - len(rows)) for rows in table]
        rest = {"lens": _i32(lens)}
    else:
        table, refs, _ = _fragmented(case)
        live = sum(1 for r in refs if r)
        holes = [p for p in range(live) if not refs[p]]
        copies = list(zip([p for p in range(live, len(refs)) if refs[p]], holes))
        to = dict(copies)
        table = [[to.get(p, p) for p in rows] for rows in table]
        refs = [r for r in refs]
        for a, b in copies:
            refs[b], refs[a] = refs[a], 0
        rest = {"live": _i32([live])}
    pool = torch.randint(0, 256, (case["layers"], len(refs), _page_bytes(case)), dtype=torch.uint8, device=DEV,
                         generator=_rng(seed, 0))
    for a, b in copies:
        pool[:, b] = pool[:, a]
    return {"pool": pool, "table": _i32(table), "refs": _i32(refs), **rest}
