"""Several answers about one image, several tokens a step: a decoder behind a
scheduled CNN block whose next words a smaller model drafts.

    python examples/draft_answers.py [--answers 4] [--steps 8]

The trunk, the decoder and its 4-bit cache are those of answer_maps.py, with
positions (``ios_rotate``).  The smaller model looks at the last word only.  In
every step it draws a small tree of words behind each answer; the decoder
attends from all of them at once to the cached tokens and their ancestors
(``ios_attn_tree``), ``ios_verify`` takes the path that stands and the word that
follows it, so that the words are distributed as the decoder's own, and
``ios_cache_keep`` moves the path into the cache.  Nothing in a step waits for
the host.  Weights are random, so the answers are too, and few drafts stand.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch

import answer_maps as A
from answer_maps import DEV, DIM, HEADS, KV, VOCAB, I, i32, stream, toks

# the certain word, two drafts behind it, and a chain behind the first of them
PARENTS, DEPTHS = [-1, 0, 0, 1, 3], [0, 1, 1, 2, 3]
TREE = len(PARENTS)


def rows(t):
    return I.ios_rows(t.data_ptr(), t.shape[0], t.stride(0))


class Decoder(A.Decoder):
    def __init__(self, channels, slots, max_tokens):
        super().__init__(channels, slots, max_tokens)
        self.rotary = I.ios_rotary(DIM)
        I.ios_rotary_freqs(self.rotary, 1e4)

    def turned(self, q, k, pos):
        qo, ko = (torch.empty(t.shape, dtype=t.dtype, device=DEV) for t in (q, k))
        I.ios_rotate(self.rotary, I.IOS_BF16, DIM, toks(q), toks(qo), HEADS, toks(k), toks(ko), KV, pos.data_ptr(), stream())
        return qo, ko

    def prompt(self, slot, x):
        n, s = x.shape[0], stream()
        seq, add, cu, pos = i32([slot]), i32([n]), i32([0, n]), i32(list(range(n)))
        I.ios_cache_reserve(self.cache, 1, seq.data_ptr(), add.data_ptr(), s)
        d = self.desc(1, n)
        size = I.ios_attn_work_bytes(d, n)
        work = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)

        def attend(layer, q, k, v):
            q, k = self.turned(q, k, pos)
            out = torch.empty_like(q)
            I.ios_cache_append(self.cache, layer, I.IOS_BF16, toks(k), toks(v), 1, seq.data_ptr(), cu.data_ptr(), s)
            I.ios_attn_prompt(d, toks(q), toks(k), toks(v), toks(out), 0, cu.data_ptr(), cu.data_ptr(), work.data_ptr(),
                              size, s)
            return out
        return self.layers(x, attend)

    def draft(self, word, rnd):
        """A tree of words behind each answer's last one, [answers][TREE], and the smaller model's probabilities there."""
        words, probs = [word], []
        for j in range(TREE):
            if j:
                words.append(torch.multinomial(probs[PARENTS[j]], 1, generator=rnd)[:, 0])
            probs.append(torch.softmax((self.out[words[j]] @ self.words).float(), 1))
        return torch.stack(words, 1), torch.stack(probs, 1).flatten(0, 1)

    def step(self, slots, word, rnd):
        """Rows that stand, [answers][TREE], their number, the words of all rows, and each answer's next word."""
        n, s = len(slots), stream()
        words, q_probs = self.draft(word, rnd)
        seqs, cu, parent = i32(slots), i32([TREE * i for i in range(n + 1)]), i32(PARENTS * n)
        pos = (self.lens[torch.tensor(slots, device=DEV)][:, None] + i32(DEPTHS)).flatten().contiguous()
        d = self.desc(n, self.max_tokens)
        size = I.ios_attn_tree_work_bytes(d, TREE * n, TREE)
        work = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
        kept = []

        def attend(layer, q, k, v):
            q, k = self.turned(q, k, pos)
            kept.append((k, v))
            out = torch.empty_like(q)
            I.ios_attn_tree(self.cache, layer, d, toks(q), toks(k), toks(v), toks(out), 0, seqs.data_ptr(), cu.data_ptr(),
                            parent.data_ptr(), TREE, work.data_ptr(), size, s)
            return out
        probs = torch.softmax((self.layers(self.out[words.flatten()], attend) @ self.words).float(), 1)
        accept, sample = (torch.rand(m, device=DEV, generator=rnd) for m in (TREE * n, n))
        tokens = words.to(torch.int32).flatten()
        path, count = torch.empty(n, TREE, dtype=torch.int32, device=DEV), torch.empty(n, dtype=torch.int32, device=DEV)
        following = torch.empty(n, dtype=torch.int32, device=DEV)
        v = I.ios_verify_desc(I.IOS_F32, n, VOCAB, TREE)
        size = I.ios_verify_work_bytes(v)
        scratch = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
        I.ios_verify(v, rows(probs), rows(q_probs), tokens.data_ptr(), parent.data_ptr(), cu.data_ptr(), accept.data_ptr(),
                     sample.data_ptr(), path.data_ptr(), count.data_ptr(), following.data_ptr(), scratch.data_ptr(), size, s)
        I.ios_cache_reserve(self.cache, n, seqs.data_ptr(), count.data_ptr(), s)
        for layer, (k, val) in enumerate(kept):
            I.ios_cache_keep(self.cache, layer, I.IOS_BF16, toks(k), toks(val), n, seqs.data_ptr(), path.data_ptr(), TREE,
                             count.data_ptr(), s)
        return path, count, tokens, following


def answers(count=4, steps=8):
    """The words of every answer, the number that stood in each step [steps][count], and the decoder."""
    image = A.feature_map().to(torch.bfloat16)
    dec = Decoder(image.shape[1], 1 + count, image.shape[0] + steps * TREE + 1)
    rnd = torch.Generator(DEV).manual_seed(1)
    last = dec.prompt(0, image @ dec.embed)[-1:]
    kids = list(range(1, 1 + count))
    parents, children = i32([0] * count), i32(kids)
    I.ios_cache_fork(dec.cache, count, parents.data_ptr(), children.data_ptr(), stream())
    word = (last @ dec.words).float().topk(count).indices[0]
    done = []
    for _ in range(steps):
        path, stood, tokens, following = dec.step(kids, word, rnd)
        done.append((path, stood, tokens))
        word = following.long()
    if I.ios_cache_status(dec.cache, stream()):
        raise RuntimeError("the cache ran out of pages")
    out = [[] for _ in kids]
    for path, stood, tokens in done:
        for i in range(count):
            out[i] += tokens[path[i, :int(stood[i])].long()].tolist()
    return out, [stood.tolist() for _, stood, _ in done], dec


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--answers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    ids, stood, _ = answers(a.answers, a.steps)
    for i, row in enumerate(ids):
        print(f"answer {i}: {row}")
    print("words a step:", stood)
