"""Several answers about one image, token by token: a scheduled CNN block, and a
small decoder that reads its feature map.

    python examples/answer_maps.py [--answers 4] [--tokens 16]

The Inception block runs under the greedy schedule (``ios_run``); its 35x35 map
becomes a prompt of 1225 tokens, which every layer attends over once
(``ios_attn_prompt``) and keeps in the 4-bit cache (``ios_cache_append``).  The
answers are forks of that sequence (``ios_cache_fork``): they share its pages
until they write (``ios_cache_reserve`` copies the last one for each), and take
one token at a time (``ios_attn_cache``).  Weights are random, so the answers
are too; projections and the choice of tokens are plain torch.
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import paper_2011_01302_amd as I
import workloads as W

DEV, LAYERS, HEADS, KV, DIM, PAGE, VOCAB = "cuda:0", 2, 8, 2, 64, 32, 512
WIDTH = HEADS * DIM


def stream():
    return torch.cuda.current_stream().cuda_stream


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def toks(t):
    return I.ios_tokens(t.data_ptr(), t.shape[0], t.stride(0), t.stride(1))


def feature_map():
    """The Inception block's output on a synthetic image, as tokens [1225][channels]."""
    spec, ten = W.make("inception", 1, 0)
    g = I.Graph(spec, ten)
    o = I.ios_sched_opts_default()
    o.mode = I.IOS_SCHED_GREEDY
    q, _ = I.ios_schedule(g.handle, o)
    shapes = W.infer_shapes(spec)
    ins = [torch.from_numpy(np.ascontiguousarray(ten[t["name"]])).to(DEV) for t in spec["inputs"]]
    outs = [torch.empty((1,) + tuple(shapes[n]), device=DEV) for n in spec["outputs"]]
    I.ios_run(g.handle, q, [t.data_ptr() for t in ins], [t.data_ptr() for t in outs], stream())
    torch.cuda.synchronize()
    I.ios_schedule_destroy(q)
    g.close()
    return torch.cat([t.flatten(2) for t in outs], 1)[0].t().contiguous()


class Decoder:
    """Layers of attention and a projection, their cache, and the words."""

    def __init__(self, channels, slots, max_tokens):
        rnd = torch.Generator().manual_seed(0)
        draw = lambda *s: (torch.randn(*s, generator=rnd) / math.sqrt(s[0])).to(torch.bfloat16).to(DEV)  # noqa: E731
        self.embed, self.words, self.out = draw(channels, WIDTH), draw(WIDTH, VOCAB), draw(VOCAB, WIDTH)
        self.qkv = [draw(WIDTH, (HEADS + 2 * KV) * DIM) for _ in range(LAYERS)]
        self.proj = [draw(WIDTH, WIDTH) for _ in range(LAYERS)]
        c = self.cache = I.ios_cache()
        c.layers, c.kv_heads, c.head_dim, c.page_tokens = LAYERS, KV, DIM, PAGE
        c.slots, c.row = slots, -(-max_tokens // PAGE)
        c.pages = c.row + 2 * slots + (slots - 1) * (c.row // 4)
        self.pool = torch.empty(LAYERS, c.pages, I.ios_cache_page_bytes(c), dtype=torch.uint8, device=DEV)
        self.refs, self.lens = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (c.pages, slots))
        self.table = torch.full((slots, c.row), -1, dtype=torch.int32, device=DEV)
        self.work = torch.zeros(I.ios_cache_work_bytes(c), dtype=torch.uint8, device=DEV)
        c.pool, c.refs, c.table, c.lens, c.work = (t.data_ptr() for t in
                                                   (self.pool, self.refs, self.table, self.lens, self.work))
        self.max_tokens = max_tokens

    def desc(self, seqs, keys):
        d = I.ios_attn_desc()
        d.dtype, d.heads, d.kv_heads, d.head_dim, d.seqs = I.IOS_BF16, HEADS, KV, DIM, seqs
        d.causal, d.max_keys, d.scale = 1, keys, 1 / math.sqrt(DIM)
        return d

    def layers(self, x, attend):
        """x [tokens][WIDTH] through every layer; attend(layer, q, k, v) is its attention."""
        for i in range(LAYERS):
            y = (torch.nn.functional.normalize(x.float(), dim=-1) * math.sqrt(WIDTH)).to(x.dtype) @ self.qkv[i]
            q, k, v = y.view(-1, HEADS + 2 * KV, DIM).split([HEADS, KV, KV], 1)
            x = x + attend(i, q, k, v).reshape(-1, WIDTH) @ self.proj[i]
        return x

    def prompt(self, slot, x):
        n, s = x.shape[0], stream()
        seq, add, cu = i32([slot]), i32([n]), i32([0, n])
        I.ios_cache_reserve(self.cache, 1, seq.data_ptr(), add.data_ptr(), s)
        d = self.desc(1, n)
        size = I.ios_attn_work_bytes(d, n)
        work = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)

        def attend(layer, q, k, v):
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            I.ios_cache_append(self.cache, layer, I.IOS_BF16, toks(k), toks(v), 1, seq.data_ptr(), cu.data_ptr(), s)
            I.ios_attn_prompt(d, toks(q), toks(k), toks(v), toks(out), 0, cu.data_ptr(), cu.data_ptr(),
                              work.data_ptr(), size, s)
            return out
        return self.layers(x, attend)

    def step(self, slots, x):
        """One token for every slot."""
        n, s = len(slots), stream()
        seqs, add, cu = i32(slots), i32([1] * n), i32(list(range(n + 1)))
        I.ios_cache_reserve(self.cache, n, seqs.data_ptr(), add.data_ptr(), s)
        d = self.desc(n, self.max_tokens)
        size = I.ios_attn_work_bytes(d, n)
        work = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)

        def attend(layer, q, k, v):
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            I.ios_cache_append(self.cache, layer, I.IOS_BF16, toks(k), toks(v), n, seqs.data_ptr(), cu.data_ptr(), s)
            I.ios_attn_cache(self.cache, layer, d, toks(q), toks(out), 0, seqs.data_ptr(), work.data_ptr(), size, s)
            return out
        return self.layers(x, attend)


def answers(count=4, tokens=16):
    """Token ids [count][tokens], and the pages in use with every answer and after all but the first have gone."""
    image = feature_map().to(torch.bfloat16)
    dec = Decoder(image.shape[1], 1 + count, image.shape[0] + tokens + 1)
    last = dec.prompt(0, image @ dec.embed)[-1:]
    kids = list(range(1, 1 + count))
    parents, children = i32([0] * count), i32(kids)
    I.ios_cache_fork(dec.cache, count, parents.data_ptr(), children.data_ptr(), stream())
    # each answer starts with another of the likeliest words
    word = (last @ dec.words).float().topk(count).indices[0]
    out = [word]
    for _ in range(tokens - 1):
        x = dec.step(kids, dec.out[word])
        word = (x @ dec.words).float().argmax(-1)
        out.append(word)
    live = [torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2)]
    I.ios_cache_compact(dec.cache, live[0].data_ptr(), stream())
    I.ios_cache_free(dec.cache, count - 1, children[1:].data_ptr(), stream())
    I.ios_cache_compact(dec.cache, live[1].data_ptr(), stream())
    if I.ios_cache_status(dec.cache, stream()):
        raise RuntimeError("the cache ran out of pages")
    return torch.stack(out, 1).tolist(), [int(t) for t in live], dec


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--answers", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=16)
    a = ap.parse_args()
    ids, pages, _ = answers(a.answers, a.tokens)
    for i, row in enumerate(ids):
        print(f"answer {i}: {row}")
    print(f"pages in use: {pages[0]} with {a.answers} answers, {pages[1]} with one")
