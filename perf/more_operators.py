"""Several tokens a step for the decoder behind a CNN trunk, as cases that can
be timed and checked: the rotation of queries and keys by their positions, keys
rotated on their way into the paged 4-bit cache, attention of a tree of drafted
tokens over that cache, the check of the drafts against the model's
probabilities, and the accepted ones kept in the cache.

One step of an answer: a small model drafts a tree of tokens behind the last
one, every layer rotates the queries and keys of the tree, attends from each
draft to the cached tokens and to its ancestors, the probabilities that come out
say which path of the tree stands and which token follows it, and the path's
keys and values go into the cache.  Prompts and single tokens go in without a
tree.

``run`` computes an operator in elementary torch operations where ``own`` is
false, and through the library's entry points where it is true.

Rotation.  Pair i of a head's first ``rot`` values, (i, i + rot / 2) or
(2 i, 2 i + 1), at position t:

    g   = min(max((original f_i / 2 pi - low) / (high - low), 0), 1),  f_i = base^(-2 i / rot)
    w_i = f_i (g + (1 - g) / factor), or f_i / factor where original = 0      (64 bits)
    c   = f32(amplitude cos(t w_i)),  s = f32(amplitude sin(t w_i))           (64 bits, rounded once)
    a'  = f32(a c) - f32(b s),  b' = f32(a s) + f32(b c)                      (32 bits), rounded to the type

The 4-bit format, for 32 consecutive values x of one head's key or value (all
steps in float32, each rounded once):

    x   = min(max(x, -61440), 61440)
    z   = f16(min x),  s = f16((max x - min x) * f32(1 / 15))
    c_i = min(max(round_half_even((x_i - z) / s), 0), 15), 0 where s = 0
    the value that is held: z + s c_i

The check of drafts.  Row 0 of a sequence is the token that is certain; it is
the first node.  The children of the node are tried in their order: child x
stands where accept_x S q(x) < max(p(x) - C q(x), 0), p the model's and q the
draft's probabilities in the node's row, with C = 0 and S = 1 at first; where it
does not, C grows by S, and S becomes sum_t max(p(t) - C q(t), 0).  A child that
stands is the next node.  Drafts without probabilities are certain ones: x stands
where accept_x S < p(x), and if not S shrinks by p(x) and x is left out.  The
next token is the first whose running sum of max(p - C q, 0) (of p without
what was left out) passes ``sample`` times the whole sum.  In 64 bits.
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
        # the newest tokens of a few answers, far into their sequences: launch latency
        {"name": "rotate_tokens", "op": "rotate", "dtype": "f16", "heads": 8, "kv_heads": 2, "head_dim": 64, "rot": 64,
         "inter": False, "base": 1e4, "factor": 1.0, "original": 0, "lens": "1," * 15 + "1", "start": 60000},
        # a long prompt and a short one behind it, every pair beside its partner, positions scaled eight times beyond
        # what the model saw
        {"name": "rotate_prompts", "op": "rotate", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "rot": 128, "inter": False, "base": 5e5, "factor": 8.0, "original": 8192, "lens": "16384,1225", "start": 0},
        # the newest token of every sequence of a batch, its query rotated in the same call
        {"name": "append_tokens", "op": "append", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "rot": 128, "inter": False, "base": 1e4, "factor": 4.0, "original": 0, "page": 64,
         "lens": ",".join(str(64 + 97 * i) for i in range(32)), "new": ",".join(["1"] * 32)},
        # maps of every size as prompts, half of each head turned, neighbours as pairs
        {"name": "append_maps", "op": "append", "dtype": "f16", "heads": 16, "kv_heads": 8, "head_dim": 64, "rot": 32,
         "inter": True, "base": 1e4, "factor": 1.0, "original": 0, "page": 64,
         "lens": "3025,1764,12289,1225,784,64", "new": "3025,1764,12289,1225,784,49"},
        # one answer about a 28x28 map, in the trunk's own type, a small tree
        {"name": "tree_28x28", "op": "tree", "dtype": "f32", "heads": 8, "kv_heads": 2, "head_dim": 64, "page": 32,
         "lens": "785", "drafts": "7"},
        # a batch of answers over maps of every size, trees of every size, a sequence without drafts among them
        {"name": "tree_maps", "op": "tree", "dtype": "f16", "heads": 16, "kv_heads": 4, "head_dim": 96, "page": 32,
         "lens": "65,785,1226,1765,3026,1,33,129,801,1240,1799,3100,97,790,1300,2048",
         "drafts": "9,13,1,33,5,8,8,13,21,0,64,5,7,13,12,3"},
        # one sequence with a long cache and a wide tree
        {"name": "tree_one_long", "op": "tree", "dtype": "bf16", "heads": 16, "kv_heads": 2, "head_dim": 128,
         "page": 128, "lens": "131072", "drafts": "32"},
        # a full batch of long sequences
        {"name": "tree_batch", "op": "tree", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64,
         "lens": ",".join(str(8192 + 769 * i) for i in range(32)), "drafts": ",".join(["16"] * 32)},
        # chains drawn from a small model with a large vocabulary, a batch of answers
        {"name": "verify_chains", "op": "verify", "dtype": "f32", "vocab": 131072, "drafts": ",".join(["6"] * 32),
         "shape": "chain", "given": True},
        # one tree of likely tokens for a vocabulary of an odd size
        {"name": "verify_tree", "op": "verify", "dtype": "bf16", "vocab": 32003, "drafts": "25", "shape": "tree",
         "given": False},
        # the accepted tokens of a few trees
        {"name": "keep_few", "op": "keep", "dtype": "f16", "kv_heads": 2, "head_dim": 64, "page": 32,
         "lens": "786,1230,1765,3030", "kept": "1,4,0,5", "drafts": 13},
        # those of a large batch
        {"name": "keep_batch", "op": "keep", "dtype": "bf16", "kv_heads": 8, "head_dim": 128, "page": 64,
         "lens": ",".join(str(40 + 29 * i) for i in range(256)), "kept": ",".join(str(1 + 5 * i % 9) for i in range(256)),
         "drafts": 16},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(values):
    return ",".join(map(str, values))


def draw(rng: random.Random):
    op = rng.choice(["rotate", "append", "append", "tree", "tree", "tree", "verify", "verify", "keep"])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 2, 4, 5, 8] if kv < 8 else [1, 2, 4])
    page = rng.choice([32, 64, 128, 256])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    dim = rng.choice([32, 64, 96, 128])
    if op in ("rotate", "append"):
        if op == "rotate":
            dim = rng.choice([8, 32, 40, 64, 80, 96, 128])
        rot = dim if rng.random() < 0.5 else 2 * rng.randint(1, dim // 2)
        c = {"op": op, "dtype": dtype, "heads": heads, "kv_heads": kv, "head_dim": dim, "rot": rot,
             "inter": rng.random() < 0.5, "base": rng.choice([1e4, 5e5, 1e6]), "factor": rng.choice([1.0, 2.5, 8.0, 32.0]),
             "original": rng.choice([0, 2048, 4096, 8192])}
        if op == "rotate":
            lens = [_log(rng, 1, 4000) for _ in range(_log(rng, 1, 4))]
            return {**c, "lens": _text(lens), "start": rng.choice([0, _log(rng, 1, 1000000)])}
        lens = [_log(rng, 1, 2500) for _ in range(_log(rng, 1, 6))]
        new = [1] * len(lens) if rng.random() < 0.4 else [_log(rng, 1, m) for m in lens]
        return {**c, "page": page, "lens": _text(lens), "new": _text(new)}
    if op == "tree":
        lens = [_log(rng, 1, 40000) for _ in range(_log(rng, 1, 32))]
        drafts = [rng.randint(1, rng.choice([2, 8, 16, 64])) for _ in lens]
        while heads * dim * sum(m * n for m, n in zip(lens, drafts)) > 5e10:      # less than the largest listed one
            lens = [(m + 1) // 2 for m in lens]
        return {"op": op, "dtype": dtype, "heads": heads, "kv_heads": kv, "head_dim": dim, "page": page,
                "lens": _text(lens), "drafts": _text(drafts)}
    if op == "verify":
        vocab, n, shape = _log(rng, 50, 131072), _log(rng, 1, 32), rng.choice(["chain", "tree"])
        drafts = [rng.randint(1, 9 if shape == "chain" else 40) for _ in range(n)]
        while sum(drafts) * vocab > 2.4e7:
            vocab = (vocab + 1) // 2
        return {"op": op, "dtype": dtype, "vocab": vocab, "drafts": _text(drafts), "shape": shape,
                "given": rng.random() < 0.5}
    n, drafts = _log(rng, 1, 200), rng.randint(1, 64)
    kept = [rng.randint(0, min(drafts, 12)) for _ in range(n)]
    return {"op": op, "dtype": dtype, "kv_heads": kv, "head_dim": dim, "page": page,
            "lens": _text([m + _log(rng, 1, 3000) for m in kept]), "kept": _text(kept), "drafts": drafts}


def _ints(text):
    return [int(v) for v in text.split(",")]


def _pages(tokens, page):
    return -(-tokens // page)


def _size(case):
    return 4 if case["dtype"] == "f32" else 2


def work(case):
    op, size = case["op"], _size(case)
    if op == "rotate":
        values = sum(_ints(case["lens"])) * (case["heads"] + case["kv_heads"]) * case["head_dim"]
        return {"bytes": 2 * size * values, "flops": 3 * values * case["rot"] // case["head_dim"]}
    if op in ("append", "keep"):      # the input, the cache written and read, the values in 32 bits; queries in and out
        new = sum(_ints(case["new" if op == "append" else "kept"]))
        values, turned = 2 * new * case["kv_heads"] * case["head_dim"], new * case.get("heads", 0) * case["head_dim"]
        return {"bytes": (size + 4) * values + 2 * values * 5 // 8 + 2 * size * turned, "flops": 8 * values + 3 * turned}
    if op == "tree":
        lens, drafts = _ints(case["lens"]), _ints(case["drafts"])
        h, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
        return {"bytes": sum(m for m, n in zip(lens, drafts) if n) * kv * 2 * (d // 2 + 4 * d // GROUP) +
                size * sum(drafts) * d * 2 * (h + kv),
                "flops": 4 * d * h * sum(n * (m + 1) for m, n in zip(lens, drafts))}
    values = len(_ints(case["drafts"])) * case["vocab"] * (2 if case["given"] else 1)      # the row of the last node
    return {"bytes": size * values, "flops": 3 * values}


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


def _positions(case):
    """Sequences that start one after another, at positions far apart."""
    return _i32([case["start"] + 1000 * i + j for i, m in enumerate(_ints(case["lens"])) for j in range(m)])


def _scaling(case):
    """base, factor, original, low, high of the rotation, and its amplitude."""
    return case["base"], case["factor"], float(case["original"]), 1.0, 32.0 if case["inter"] else 4.0


def _amplitude(case):
    return 1.0 if case["original"] == 0 else 1.0 + 0.125 * round(math.log(case["factor"]))


def _parents(count, shape, rng):
    """Row 0 is the last certain token, the others are drafted behind it."""
    if shape == "chain":
        return [j - 1 for j in range(count)]
    return [-1] + [rng.randint(max(0, j - 9), j - 1) for j in range(1, count)] if count else []


def _trees(case, seed):
    rng = random.Random(seed)
    return [_parents(n, case.get("shape", "tree"), rng) for n in _ints(case["drafts"])]


def _distributions(case, seed):
    """The model's and the draft's probabilities behind every row, the drafted tokens, and the random numbers."""
    rows = sum(_ints(case["drafts"]))
    logits = 4.0 * torch.randn(rows, case["vocab"], generator=_rng(seed, 0), device=DEV)
    p = torch.softmax(logits, 1).to(DTYPES[case["dtype"]])
    logits += torch.randn(rows, case["vocab"], generator=_rng(seed, 1), device=DEV)
    q = torch.softmax(logits, 1).to(DTYPES[case["dtype"]])
    before, at = [], 0
    for tree in _trees(case, seed):
        before += [at + max(j, 0) for j in tree]
        at += len(tree)
    tokens = torch.multinomial(q[torch.tensor(before, device=DEV)].float(), 1, generator=_rng(seed, 2)).flatten()
    accept = torch.rand(rows, generator=_rng(seed, 3), device=DEV)
    sample = torch.rand(len(_ints(case["drafts"])), generator=_rng(seed, 4), device=DEV)
    return p, q, tokens.to(torch.int32), accept, sample


def _paths(case, seed):
    """Rows of the accepted drafts, as the check leaves them: [sequences][drafts], -1 behind them."""
    rng, n = random.Random(seed), case["drafts"]
    return [[i * n + j for j in [0] * (m > 0) + sorted(rng.sample(range(1, n), m - 1) if m > 1 else [])] + [-1] * (n - m)
            for i, m in enumerate(_ints(case["kept"]))]


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


def _dtype(case):
    import paper_2011_01302_amd as I
    return {"f32": I.IOS_F32, "f16": I.IOS_F16, "bf16": I.IOS_BF16}[case["dtype"]]


def _cache(case, lens, seed):
    """The library's description of a cache of one layer, and the tensors that it points to."""
    import paper_2011_01302_amd as I
    table, refs = _shuffled_table(case, lens, seed)
    st = {"refs": _i32(refs), "table": _i32(table), "cached": _i32(lens), "dtype": _dtype(case)}
    c = I.ios_cache()
    c.layers, c.kv_heads, c.head_dim, c.page_tokens = 1, case["kv_heads"], case["head_dim"], case["page"]
    c.pages, c.slots, c.row = len(refs), len(table), len(table[0])
    st["pool"] = torch.zeros(1, len(refs), I.ios_cache_page_bytes(c), dtype=torch.uint8, device=DEV)
    st["cache_work"] = torch.zeros(I.ios_cache_work_bytes(c), dtype=torch.uint8, device=DEV)
    c.pool, c.refs, c.table, c.lens = (st[n].data_ptr() for n in ("pool", "refs", "table", "cached"))
    c.work = st["cache_work"].data_ptr()
    st["cache"] = c
    return st


def _rotary(case):
    """The library's description of a rotation."""
    import paper_2011_01302_amd as I
    r = I.ios_rotary()
    r.dim, r.interleaved, r.amplitude = case["rot"], int(case["inter"]), _amplitude(case)
    I.ios_rotary_freqs(r, *_scaling(case))
    return r


def _tokens(t):
    """[tokens][heads][head_dim], the last dimension contiguous."""
    import paper_2011_01302_amd as I
    return I.ios_tokens(t.data_ptr(), t.shape[0], t.stride(0), t.stride(1))


def _fill_cache(st, case, lens, seed):
    """Sequences that are cached already: in the library's cache, or as codes, scales and zero points, padded to the
    longest."""
    if own:
        import paper_2011_01302_amd as I
        st.update(_cache(case, lens, seed))
    else:
        n, kv, groups, most = len(lens), case["kv_heads"], case["head_dim"] // GROUP, max(lens)
        st["codes"] = torch.zeros(n, 2, kv, most, groups, GROUP, dtype=torch.uint8, device=DEV)
        st["scales"], st["zeros"] = (torch.zeros(n, 2, kv, most, groups, 1, dtype=torch.float16, device=DEV)
                                     for _ in range(2))
    for i, m in enumerate(lens):
        kv = _kv(case, m, seed, 10 + i)
        if own:
            one = _i32([i, 0, m])
            I.ios_cache_append(st["cache"], 0, st["dtype"], _tokens(kv[:, 0]), _tokens(kv[:, 1]), 1,
                               one.data_ptr(), one[1:].data_ptr(), _stream())
        else:
            for held, part in zip((st["codes"], st["scales"], st["zeros"]), _quantised(kv)):
                held[i, :, :, :m] = part.movedim(0, 2)


def prepare(case, seed):
    st, op = {"case": case}, case["op"]
    if op == "rotate":
        joint = torch.cat([_queries(case, sum(_ints(case["lens"])), seed),
                           _kv(case, sum(_ints(case["lens"])), seed, 3).flatten(1, 2)], 1)     # one projection's output
        st["q"], st["k"] = joint[:, :case["heads"]], joint[:, case["heads"]:case["heads"] + case["kv_heads"]]
        st["pos"] = _positions(case)
        if own:
            st["rotary"], st["dtype"] = _rotary(case), _dtype(case)
    elif op == "append":
        lens, new = _ints(case["lens"]), _ints(case["new"])
        kv = _kv(case, sum(new), seed, 3)
        st["q"], st["k"], st["v"] = _queries(case, sum(new), seed), kv[:, 0], kv[:, 1]
        st["seqs"], st["cu"], st["lens"] = _i32(list(range(len(lens)))), _i32(_offsets(new)), _i32(lens)
        if own:
            st.update(_cache(case, lens, seed))
            st["rotary"] = _rotary(case)
    elif op == "tree":
        lens, trees = _ints(case["lens"]), _trees(case, seed)
        rows = sum(map(len, trees))
        kv = _kv(case, rows, seed, 3)
        st["q"], st["k"], st["v"] = _queries(case, rows, seed), kv[:, 0], kv[:, 1]
        st["seqs"], st["lens"], st["most"] = _i32(list(range(len(lens)))), _i32(lens), max(map(len, trees))
        st["cu"], st["parent"] = _i32(_offsets(map(len, trees))), _i32([j for t in trees for j in t])
        _fill_cache(st, case, lens, seed)
        if own:
            import paper_2011_01302_amd as I
            d = st["desc"] = I.ios_attn_desc()
            d.dtype, d.heads, d.kv_heads, d.head_dim = st["dtype"], case["heads"], case["kv_heads"], case["head_dim"]
            d.seqs, d.max_keys, d.scale = len(lens), max(lens), 1.0 / math.sqrt(case["head_dim"])
            n = st["work_bytes"] = I.ios_attn_tree_work_bytes(d, rows, st["most"])
            st["work"] = torch.zeros(max(n, 16), dtype=torch.uint8, device=DEV)
    elif op == "verify":
        trees = _trees(case, seed)
        st["p"], st["q"], st["tokens"], st["accept"], st["sample"] = _distributions(case, seed)
        st["cu"], st["parent"] = _i32(_offsets(map(len, trees))), _i32([j for t in trees for j in t])
        st["most"] = max(map(len, trees))
        if own:
            import paper_2011_01302_amd as I
            d = st["desc"] = I.ios_verify_desc()
            d.dtype, d.seqs, d.vocab, d.max_drafts = _dtype(case), len(trees), case["vocab"], st["most"]
            n = st["work_bytes"] = I.ios_verify_work_bytes(d)
            st["work"] = torch.zeros(max(n, 16), dtype=torch.uint8, device=DEV)
    else:
        lens, kept, paths = _ints(case["lens"]), _ints(case["kept"]), _paths(case, seed)
        kv = _kv(case, len(lens) * case["drafts"], seed, 3)
        st["k"], st["v"] = kv[:, 0], kv[:, 1]
        st["seqs"], st["path"], st["count"] = _i32(list(range(len(lens)))), _i32(paths), _i32(kept)
        st["cu"] = _i32(_offsets(kept))
        if own:
            st.update(_cache(case, lens, seed))
    return st


# ---------------------------------------------------------------- one pass

def _stream():
    return torch.cuda.current_stream().cuda_stream


def run(st):
    op = st["case"]["op"]
    if own:
        return {"rotate": _own_rotate, "append": _own_append, "tree": _own_tree, "verify": _own_verify,
                "keep": _own_keep}[op](st)
    return {"rotate": _plain_rotate, "append": _plain_append, "tree": _plain_tree, "verify": _plain_verify,
            "keep": _plain_keep}[op](st)


def _like(t):
    return torch.empty(t.shape, dtype=t.dtype, device=DEV)


def _own_rotate(st):
    import paper_2011_01302_amd as I
    q, k, case = st["q"], st["k"], st["case"]
    qo, ko = _like(q), _like(k)
    I.ios_rotate(st["rotary"], st["dtype"], case["head_dim"], _tokens(q), _tokens(qo), case["heads"], _tokens(k),
                 _tokens(ko), case["kv_heads"], st["pos"].data_ptr(), _stream())
    return qo, ko


def _read_back(st, rows):
    import paper_2011_01302_amd as I
    ko = torch.empty(rows, *st["k"].shape[1:], dtype=torch.float32, device=DEV)
    vo = torch.empty_like(ko)
    I.ios_cache_read(st["cache"], 0, I.IOS_F32, _tokens(ko), _tokens(vo), st["seqs"].shape[0], st["seqs"].data_ptr(),
                     st["cu"].data_ptr(), _stream())
    return ko, vo


def _own_append(st):
    import paper_2011_01302_amd as I
    q, k, v, case = st["q"], st["k"], st["v"], st["case"]
    qo = _like(q)
    I.ios_cache_append_rotary(st["cache"], 0, st["dtype"], st["rotary"], _tokens(q), _tokens(qo), case["heads"],
                              _tokens(k), _tokens(v), st["seqs"].shape[0], st["seqs"].data_ptr(), st["cu"].data_ptr(),
                              _stream())
    return qo, *_read_back(st, k.shape[0])


def _own_tree(st):
    import paper_2011_01302_amd as I
    out = _like(st["q"])
    I.ios_attn_tree(st["cache"], 0, st["desc"], _tokens(st["q"]), _tokens(st["k"]), _tokens(st["v"]), _tokens(out), 0,
                    st["seqs"].data_ptr(), st["cu"].data_ptr(), st["parent"].data_ptr(), st["most"],
                    st["work"].data_ptr(), st["work_bytes"], _stream())
    return out


def _own_verify(st):
    import paper_2011_01302_amd as I
    n, p, q = st["sample"].shape[0], st["p"], st["q"]
    path = torch.empty(n, st["most"], dtype=torch.int32, device=DEV)
    count, following = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, dtype=torch.int32, device=DEV)
    rows = lambda t: I.ios_rows(t.data_ptr(), t.shape[0], t.stride(0))  # noqa: E731
    I.ios_verify(st["desc"], rows(p), rows(q) if st["case"]["given"] else None, st["tokens"].data_ptr(),
                 st["parent"].data_ptr(), st["cu"].data_ptr(), st["accept"].data_ptr(), st["sample"].data_ptr(),
                 path.data_ptr(), count.data_ptr(), following.data_ptr(), st["work"].data_ptr(), st["work_bytes"],
                 _stream())
    return path, count, following


def _own_keep(st):
    import paper_2011_01302_amd as I
    I.ios_cache_keep(st["cache"], 0, st["dtype"], _tokens(st["k"]), _tokens(st["v"]), st["seqs"].shape[0],
                     st["seqs"].data_ptr(), st["path"].data_ptr(), st["path"].shape[1], st["count"].data_ptr(),
                     _stream())
    return _read_back(st, sum(_ints(st["case"]["kept"])))


def _frequencies(case):
    base, factor, original, low, high = _scaling(case)
    f = [base ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]
    if original:
        g = [min(max((original * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        f = [x * (a + (1.0 - a) / factor) for x, a in zip(f, g)]
    else:
        f = [x / factor for x in f]
    return torch.tensor(f, dtype=torch.float64, device=DEV)


def _rotated(case, x, pos):
    """x [tokens][heads][head_dim] at positions pos."""
    angle = pos.double()[:, None] * _frequencies(case)
    c, s = ((_amplitude(case) * t).float()[:, None] for t in (torch.cos(angle), torch.sin(angle)))
    head, tail = x[..., :case["rot"]].float(), x[..., case["rot"]:]
    if case["inter"]:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = head.chunk(2, -1)
        turned = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([turned.to(x.dtype), tail], -1)


def _plain_rotate(st):
    return tuple(_rotated(st["case"], st[n], st["pos"]) for n in ("q", "k"))


def _quantised(x):
    """Codes, scales and zero points of x [..][head_dim]."""
    x = x.float().clamp(-LIMIT, LIMIT).unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    z = lo.half()
    s = ((hi - lo) * torch.tensor(1.0 / 15.0, device=x.device)).half()
    c = torch.where(s > 0, torch.round((x - z.float()) / s.float()).clamp(0, 15), 0.0)
    return c.to(torch.uint8), s, z


def _values(c, s, z):
    return (z.float() + s.float() * c.float()).flatten(-2)


def _plain_append(st):
    """The tokens of the call are the last ones of their sequences."""
    q, k, v, cu = st["q"], st["k"], st["v"], st["cu"]
    row = torch.arange(k.shape[0], device=DEV)
    seq = torch.searchsorted(cu, row, right=True) - 1
    pos = (st["lens"] - cu[1:])[seq] + row
    return (_rotated(st["case"], q, pos), _values(*_quantised(_rotated(st["case"], k, pos))), _values(*_quantised(v)))


def _plain_keep(st):
    path = st["path"].long()
    rows = path[path >= 0]
    return _values(*_quantised(st["k"][rows])), _values(*_quantised(st["v"][rows]))


def _seen(parent, seq, at, n, most):
    """Which drafts of its sequence a row sees, [sequences][row][draft]: itself and its ancestors."""
    step = torch.zeros(n, most, most, device=DEV)
    up = parent >= 0
    step[seq[up], at[up], parent[up].long()] = 1.0
    return torch.linalg.matrix_power(step + torch.eye(most, device=DEV), 64) > 0


def _plain_tree(st):
    q, n, most, cu = st["q"], st["lens"].shape[0], st["most"], st["cu"].long()
    kvh, d = st["k"].shape[1:]
    ratio = q.shape[1] // kvh
    row = torch.arange(q.shape[0], device=DEV)
    seq = torch.searchsorted(cu, row, right=True) - 1
    at = row - cu[seq]

    def padded(x):                                     # [sequences][kv_heads][most * heads per key head][head_dim]
        y = torch.zeros(n, most, kvh, x.shape[1] // kvh, d, device=DEV)
        y[seq, at] = x.float().unflatten(1, (kvh, -1))
        return y.transpose(1, 2).flatten(2, 3).contiguous()
    held = _values(st["codes"], st["scales"], st["zeros"])
    k, v = held[:, 0], held[:, 1]
    qq, kd, vd = padded(q), padded(st["k"]), padded(st["v"])
    scale = 1.0 / math.sqrt(d)
    sc = torch.matmul(qq, k.transpose(2, 3).contiguous()) * scale
    sd = torch.matmul(qq, kd.transpose(2, 3).contiguous()) * scale
    sc.masked_fill_((torch.arange(k.shape[2], device=DEV) >= st["lens"][:, None])[:, None, None], float("-inf"))
    seen = _seen(st["parent"], seq, at, n, most).repeat_interleave(ratio, 1)[:, None]
    sd.masked_fill_(~seen, float("-inf"))
    m = torch.maximum(sc.amax(-1, keepdim=True), sd.amax(-1, keepdim=True))
    pc, pd = torch.exp(sc - m), torch.exp(sd - m)
    o = (torch.matmul(pc, v.contiguous()) + torch.matmul(pd, vd)) / (pc.sum(-1, keepdim=True) + pd.sum(-1, keepdim=True))
    return o.unflatten(2, (most, ratio)).transpose(1, 2).flatten(2, 3)[seq, at].to(q.dtype)


def _plain_verify(st):
    """Every sequence at once, draft by draft in the order of the rows: a draft is tried when its turn comes and its
    parent is the node."""
    p, q, cu, given = st["p"], st["q"], st["cu"].long(), st["case"]["given"]
    n, most, last = cu.shape[0] - 1, st["most"], p.shape[0] - 1
    here, size = torch.arange(n, device=DEV), cu[1:] - cu[:-1]
    node = torch.zeros(n, dtype=torch.long, device=DEV)
    path = torch.full((n, most), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = cu[:-1]
    count = torch.ones(n, dtype=torch.long, device=DEV)
    w = p[cu[:-1]].double()                            # what the next token is drawn from
    c, s = torch.zeros(n, 1, dtype=torch.float64, device=DEV), torch.ones(n, dtype=torch.float64, device=DEV)
    for j in range(1, most):                           # the order of the drafts is part of the definition
        row = (cu[:-1] + j).clamp(max=last)
        tried = (j < size) & (st["parent"][row] == node)
        x = st["tokens"][row].long()
        qn = q[cu[:-1] + node].double()
        need = s * st["accept"][row].double() * (qn[here, x] if given else 1.0)
        stands = tried & (need < w[here, x])
        fails = tried & ~stands
        if given:
            c = torch.where(fails[:, None], c + s[:, None], c)
            left = (p[cu[:-1] + node].double() - c * qn).clamp(min=0.0)
            s = torch.where(fails, left.sum(1), s)
            w = torch.where(fails[:, None], left, w)
        else:
            s = torch.where(fails, s - w[here, x], s)
            w[here, x] = torch.where(fails, 0.0, w[here, x])
        node = torch.where(stands, j, node)
        slot = count.clamp(max=most - 1)
        path[here, slot] = torch.where(stands, row.to(torch.int32), path[here, slot])
        count += stands
        w = torch.where(stands[:, None], p[row].double(), w)
        c, s = torch.where(stands[:, None], 0.0, c), torch.where(stands, 1.0, s)
    run_sum = torch.cumsum(w, 1)
    following = (run_sum > st["sample"].double()[:, None] * run_sum[:, -1:]).to(torch.uint8).argmax(1)
    return path, count.to(torch.int32), following.to(torch.int32)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    return {"rotate": _exact_rotate, "append": _exact_append, "tree": _exact_tree, "verify": _exact_verify,
            "keep": _exact_keep}[case["op"]](case, seed)


def _turns(case, pos):
    """Cosine and sine of every position and pair, with the amplitude."""
    base, factor, original, low, high = _scaling(case)
    pairs = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
    f = torch.exp(-math.log(base) * 2 * pairs / case["rot"])
    if original:
        own_share = ((f * original / math.tau - low) / (high - low)).clip(0, 1)
        f = f * own_share + f / factor * (1 - own_share)
    else:
        f = f / factor
    turn = torch.polar(torch.full((len(pos), len(f)), _amplitude(case), dtype=torch.float64, device=DEV),
                       torch.outer(torch.as_tensor(pos, dtype=torch.float64, device=DEV), f))
    return turn[:, None]


def _pairs(case, x):
    """The rotated part of x as complex numbers."""
    x = x[..., :case["rot"]].double()
    if not case["inter"]:
        x = x.unflatten(-1, (2, -1)).transpose(-1, -2)
    return torch.view_as_complex(x.reshape(*x.shape[:2], -1, 2).contiguous())


def _back(case, z, x):
    y = torch.view_as_real(z)
    if not case["inter"]:
        y = y.transpose(-1, -2)
    return torch.cat([y.reshape(*x.shape[:2], case["rot"]), x[..., case["rot"]:].double()], -1)


def _exact_rotate(case, seed):
    n = sum(_ints(case["lens"]))
    turn = _turns(case, _positions(case))
    q, k = _queries(case, n, seed), _kv(case, n, seed, 3)[:, 0]
    return tuple(_back(case, _pairs(case, x) * turn, x) for x in (q, k))


def _held(x):
    """The values that the 4-bit format holds for x: its scale, zero point and codes are defined in 16 and 32
    bits, their sum is exact in 64."""
    y = torch.clip(x.to(torch.float32), -LIMIT, LIMIT).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    low, high = torch.aminmax(y, dim=-1, keepdim=True)
    zero, fifteenth = low.to(torch.float16).to(torch.float32), torch.full_like(low, 1.0 / 15.0)
    step = ((high - low) * fifteenth).to(torch.float16).to(torch.float32)
    code = torch.clip(torch.round(torch.nan_to_num((y - zero) / step, 0.0, 0.0, 0.0)), 0, 15)
    return (zero.double() + step.double() * code.double()).reshape(x.shape)


def _exact_append(case, seed):
    """What goes into the cache is defined by its roundings: cosine and sine, each product and their sums to 32 bits,
    the result to the type; the queries are not."""
    lens, new = _ints(case["lens"]), _ints(case["new"])
    turn = _turns(case, [m - n + j for m, n in zip(lens, new) for j in range(n)])
    q, kv = _queries(case, sum(new), seed), _kv(case, sum(new), seed, 3)
    z, to32 = _pairs(case, kv[:, 0]), lambda t: t.to(torch.float32).to(torch.float64)  # noqa: E731
    c, s = to32(turn.real), to32(turn.imag)
    real, imag = to32(z.real * c) - to32(z.imag * s), to32(z.real * s) + to32(z.imag * c)
    k = _back(case, torch.complex(to32(real), to32(imag)), kv[:, 0])
    return _back(case, _pairs(case, q) * turn, q), _held(k.to(torch.float32).to(kv.dtype)), _held(kv[:, 1])


def _exact_keep(case, seed):
    kv = _kv(case, len(_ints(case["lens"])) * case["drafts"], seed, 3)
    rows = [r for path in _paths(case, seed) for r in path if r >= 0]
    held = _held(kv[rows])
    return held[:, 0], held[:, 1]


def _exact_tree(case, seed):
    lens, trees = _ints(case["lens"]), _trees(case, seed)
    rows, ratio = sum(map(len, trees)), case["heads"] // case["kv_heads"]
    q, new = _queries(case, rows, seed).double(), _kv(case, rows, seed, 3).double()
    out = torch.empty(q.shape, dtype=torch.float64, device=DEV)
    at = 0
    for i, (m, tree) in enumerate(zip(lens, trees)):
        kv = torch.cat([_held(_kv(case, m, seed, 10 + i)), new[at:at + len(tree)]])
        hidden = torch.ones(len(tree), m + len(tree), dtype=torch.bool)
        hidden[:, :m] = False
        for j in range(len(tree)):
            a = j
            while a >= 0:
                hidden[j, m + a] = False
                a = tree[a]
        hidden = hidden.to(DEV)
        for h in range(case["heads"]):
            w = q[at:at + len(tree), h] @ kv[:, 0, h // ratio].T / math.sqrt(case["head_dim"])
            w[hidden] = -math.inf
            out[at:at + len(tree), h] = torch.softmax(w, 1) @ kv[:, 1, h // ratio]
        at += len(tree)
    return out


def _exact_verify(case, seed):
    """Sequence by sequence, node by node."""
    p, q, tokens, accept, sample = _distributions(case, seed)
    tokens, accept, sample = tokens.tolist(), accept.tolist(), sample.tolist()
    most = max(_ints(case["drafts"]))
    paths, counts, following = [], [], []
    first = 0
    for i, tree in enumerate(_trees(case, seed)):
        node, path = 0, [first]
        while True:
            target, left = p[first + node].double(), 1.0
            drafted, taken = q[first + node].double(), 0.0
            rest, found = target, None
            for j in (j for j in range(node + 1, len(tree)) if tree[j] == node):
                x = tokens[first + j]
                share = float(drafted[x]) if case["given"] else 1.0
                if accept[first + j] * left * share < float(rest[x]):
                    found = j
                    break
                if case["given"]:
                    taken += left
                    rest = torch.relu(target - taken * drafted)
                    left = math.fsum(rest.tolist()) if len(rest) < 4096 else float(rest.sum())
                else:
                    left -= float(rest[x])
                    rest = rest.clone()
                    rest[x] = 0.0
            if found is None:
                break
            node = found
            path.append(first + node)
        sums = rest.cumsum(0)
        following.append(int(torch.searchsorted(sums, sample[i] * sums[-1:], right=True)))
        paths.append(path + [-1] * (most - len(path)))
        counts.append(len(path))
        first += len(tree)
    return _i32(paths), _i32(counts), _i32(following)
