"""Refusals of the operators that take several tokens a step (rotation, rotated
appends, attention of drafts, their check, accepted drafts kept), and the
frequencies of a rotation: all of it on the host, so without a GPU."""
import math

import numpy as np
import pytest

import paper_2011_01302_amd as I
from test_decoder_cpu import P, cache, desc, refused, toks


def rotary(**kw):
    r = I.ios_rotary(64)
    I.ios_rotary_freqs(r, 10000.0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def rows(n=10, data=P, stride=100):
    return I.ios_rows(data, n, stride)


def check(**kw):
    d = I.ios_verify_desc(I.IOS_F32, 2, 100, 5)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


# ---------------------------------------------------------------- rotation

@pytest.mark.parametrize("dim", [2, 6, 20, 64, 128])
def test_frequencies(dim):
    f = lambda *a: (lambda r: (I.ios_rotary_freqs(r, *a), np.array(r.freq[:dim // 2]))[1])(I.ios_rotary(dim))  # noqa: E731
    plain = 10000.0 ** (-2.0 * np.arange(dim // 2) / dim)
    assert np.allclose(f(10000.0), plain, rtol=1e-15)
    assert np.allclose(f(10000.0, 8.0), plain / 8, rtol=1e-15)
    turns = 4096 * plain / (2 * math.pi)
    keep = np.clip((turns - 1.5) / (32.0 - 1.5), 0, 1)
    got = f(10000.0, 8.0, 4096.0, 1.5, 32.0)
    assert np.allclose(got, plain * (keep + (1 - keep) / 8), rtol=1e-14)
    if dim == 128:
        assert (got == plain).any() and np.isclose(got, plain / 8, rtol=1e-14).any()      # both ends of the ramp


def test_frequencies_refused_leave_them_alone():
    r = rotary()
    before = list(r.freq)
    for a in ((1.0,), (0.5,), (float("nan"),), (float("inf"),), (1e4, 0.0), (1e4, -2.0), (1e4, float("nan")),
              (1e4, 1e-4), (1e4, 1.0, -1.0), (1e4, 1.0, 4096.0, 4.0, 4.0), (1e4, 1.0, 4096.0, 4.0, 1.0),
              (1e4, 1.0, float("nan"))):
        refused("IOS_E_ARG", I.ios_rotary_freqs, r, *a)
    assert list(r.freq) == before
    for dim in (0, 1, 7, 130, -2):
        refused("IOS_E_ARG", I.ios_rotary_freqs, I.ios_rotary(dim), 1e4)
    refused("IOS_E_ARG", I.ios_rotary_freqs, None, 1e4)


def broken_rotations(dim):
    bad = I.ios_rotary(64)
    I.ios_rotary_freqs(bad, 1e4)
    bad.freq[31] = float("nan")
    far = rotary()
    far.freq[0] = -1025.0
    return [None, rotary(dim=0), rotary(dim=63), rotary(dim=dim + 2), rotary(interleaved=2), rotary(reserved=1),
            rotary(amplitude=float("inf")), rotary(amplitude=float("nan")), bad, far]


def test_rotate():
    ok = dict(r=rotary(), dtype=I.IOS_BF16, dim=64, q=toks(), qo=toks(data=2 * P), h=8, k=toks(2), ko=toks(2, data=2 * P),
              kv=2, pos=P)

    def call(**kw):
        a = {**ok, **kw}
        I.ios_rotate(a["r"], a["dtype"], a["dim"], a["q"], a["qo"], a["h"], a["k"], a["ko"], a["kv"], a["pos"])
    for r in broken_rotations(64):
        refused("IOS_E_ARG", lambda r=r: call(r=r))
    refused("IOS_E_ARG", lambda: call(dtype=3))
    refused("IOS_E_ARG", lambda: call(dim=0))
    refused("IOS_E_UNSUPPORTED", lambda: call(dim=68))
    refused("IOS_E_UNSUPPORTED", lambda: call(dim=136))
    refused("IOS_E_ARG", lambda: call(dim=32))                   # the rotation is wider
    for t, heads in (("q", 8), ("qo", 8), ("k", 2), ("ko", 2)):
        refused("IOS_E_ARG", lambda t=t: call(**{t: None}))
        refused("IOS_E_ARG", lambda t=t, heads=heads: call(**{t: toks(heads, data=0)}))
        refused("IOS_E_ARG", lambda t=t, heads=heads: call(**{t: toks(heads, data=P + 8)}))
        refused("IOS_E_ARG", lambda t=t, heads=heads: call(**{t: toks(heads, ts=516)}))
        refused("IOS_E_SHAPE", lambda t=t, heads=heads: call(**{t: toks(heads, n=11)}))
    for t in ("qo", "ko"):
        refused("IOS_E_ARG", lambda t=t: call(**{t: toks(ts=0, data=2 * P)}))
        refused("IOS_E_ARG", lambda t=t: call(**{t: toks(hs=0, data=2 * P)}))
    refused("IOS_E_ARG", lambda: call(qo=toks(ts=1024)))         # in place with other strides
    refused("IOS_E_ARG", lambda: call(h=0))
    refused("IOS_E_ARG", lambda: call(kv=0))
    refused("IOS_E_ARG", lambda: call(pos=0))
    refused("IOS_E_SHAPE", lambda: call(k=toks(2, n=9), ko=toks(2, n=9)))
    call(q=toks(n=0), qo=toks(n=0), k=toks(2, n=0), ko=toks(2, n=0))       # nothing to do, nothing launched


# ---------------------------------------------------------------- the cache

def test_append_rotary():
    ok = dict(c=cache(), layer=0, dtype=I.IOS_F16, r=rotary(), q=toks(), qo=toks(data=2 * P), h=8, k=toks(2), v=toks(2),
              n=1, seqs=P, cu=P)

    def call(**kw):
        a = {**ok, **kw}
        I.ios_cache_append_rotary(a["c"], a["layer"], a["dtype"], a["r"], a["q"], a["qo"], a["h"], a["k"], a["v"], a["n"],
                                  a["seqs"], a["cu"])
    for r in broken_rotations(64):
        refused("IOS_E_ARG", lambda r=r: call(r=r))
    refused("IOS_E_ARG", lambda: call(c=cache(head_dim=32)))     # the rotation is wider
    refused("IOS_E_ARG", lambda: call(layer=2))
    refused("IOS_E_ARG", lambda: call(dtype=-1))
    refused("IOS_E_ARG", lambda: call(q=None))
    refused("IOS_E_ARG", lambda: call(qo=None))
    refused("IOS_E_ARG", lambda: call(h=0))
    refused("IOS_E_ARG", lambda: call(qo=toks(hs=0, data=2 * P)))
    refused("IOS_E_ARG", lambda: call(qo=toks(ts=1024)))
    refused("IOS_E_SHAPE", lambda: call(q=toks(n=9), qo=toks(n=9)))
    refused("IOS_E_SHAPE", lambda: call(v=toks(2, n=9)))
    refused("IOS_E_ARG", lambda: call(n=5))
    refused("IOS_E_ARG", lambda: call(n=-1))
    refused("IOS_E_ARG", lambda: call(seqs=0))
    refused("IOS_E_ARG", lambda: call(cu=0))
    refused("IOS_E_ARG", lambda: call(c=cache(table=0)))
    refused("IOS_E_UNSUPPORTED", lambda: call(c=cache(page_tokens=48)))
    call(n=0)
    none = toks(2, n=0)
    call(q=None, qo=None, k=none, v=none)


def test_keep():
    ok = dict(c=cache(), layer=0, dtype=I.IOS_F16, k=toks(2), v=toks(2), n=1, seqs=P, path=P, most=5, count=P)

    def call(**kw):
        a = {**ok, **kw}
        I.ios_cache_keep(a["c"], a["layer"], a["dtype"], a["k"], a["v"], a["n"], a["seqs"], a["path"], a["most"], a["count"])
    for most in (0, -1, 65):
        refused("IOS_E_ARG", lambda most=most: call(most=most))
    for name in ("seqs", "path", "count"):
        refused("IOS_E_ARG", lambda name=name: call(**{name: 0}))
    refused("IOS_E_ARG", lambda: call(layer=-1))
    refused("IOS_E_ARG", lambda: call(dtype=3))
    refused("IOS_E_ARG", lambda: call(n=5))
    refused("IOS_E_ARG", lambda: call(k=toks(2, ts=4)))
    refused("IOS_E_SHAPE", lambda: call(v=toks(2, n=9)))
    refused("IOS_E_ARG", lambda: call(c=cache(pool=0)))
    call(n=0, seqs=0, path=0, count=0)


# ---------------------------------------------------------------- attention of drafts

def test_tree():
    ok = dict(c=cache(), layer=0, d=desc(), q=toks(), k=toks(2), v=toks(2), out=toks(), seqs=P, cu=P, parent=P, most=8,
              work=0, size=0)

    def call(**kw):
        a = {**ok, **kw}
        I.ios_attn_tree(a["c"], a["layer"], a["d"], a["q"], a["k"], a["v"], a["out"], 0, a["seqs"], a["cu"], a["parent"],
                        a["most"], a["work"], a["size"])
    for most in (0, -3, 65):
        refused("IOS_E_ARG", lambda most=most: call(most=most))
        refused("IOS_E_ARG", I.ios_attn_tree_work_bytes, desc(), 10, most)
    refused("IOS_E_ARG", I.ios_attn_tree_work_bytes, desc(), -1, 8)
    refused("IOS_E_SHAPE", lambda: call(d=desc(kv_heads=4)))
    refused("IOS_E_SHAPE", lambda: call(d=desc(head_dim=32)))
    refused("IOS_E_SHAPE", lambda: call(d=desc(heads=9)))
    refused("IOS_E_ARG", lambda: call(d=desc(scale=float("nan"))))
    refused("IOS_E_ARG", lambda: call(layer=2))
    for name in ("seqs", "cu", "parent"):
        refused("IOS_E_ARG", lambda name=name: call(**{name: 0}))
    for t, heads in (("q", 8), ("k", 2), ("v", 2), ("out", 8)):
        refused("IOS_E_ARG", lambda t=t: call(**{t: None}))
        refused("IOS_E_ARG", lambda t=t, heads=heads: call(**{t: toks(heads, data=P + 8)}))
        refused("IOS_E_SHAPE", lambda t=t, heads=heads: call(**{t: toks(heads, n=11)}))
    refused("IOS_E_ARG", lambda: call(out=toks(ts=0)))
    refused("IOS_E_ARG", lambda: call(c=cache(lens=0)))
    refused("IOS_E_UNSUPPORTED", lambda: call(d=desc(heads=8192), most=64))
    one = desc(seqs=1, max_keys=1 << 17)
    need = I.ios_attn_tree_work_bytes(one, 10, 8)
    assert need > 0                            # few rows, many keys: the work is spread
    refused("IOS_E_ARG", lambda: call(d=one, work=P, size=need - 1))
    refused("IOS_E_ARG", lambda: call(d=one, work=P + 4, size=need))
    call(q=toks(n=0), k=toks(2, n=0), v=toks(2, n=0), out=toks(n=0))
    assert I.ios_attn_tree_work_bytes(desc(seqs=1, max_keys=64), 10, 8) == 0


def test_tree_refuses_the_same_sizes_in_both_calls():
    """Rows and heads that no launch takes are refused before a workspace is allocated for them."""
    def call(d, n, most):
        I.ios_attn_tree(cache(), 0, d, toks(n=n), toks(2, n=n), toks(2, n=n), toks(n=n), 0, P, P, P, most, 0, 0)
    most_rows = 2 ** 25 - 1                    # of all heads, as documented
    for d, n, most in ((desc(heads=8192), 10, 64), (desc(heads=1024), 10, 64), (desc(heads=8), most_rows // 8 + 1, 8),
                       (desc(heads=16384), 2048, 3)):
        refused("IOS_E_UNSUPPORTED", I.ios_attn_tree_work_bytes, d, n, most)
        refused("IOS_E_UNSUPPORTED", lambda d=d, n=n, most=most: call(d, n, most))
    for d, n, most in ((desc(heads=1022), 10, 64), (desc(heads=8), most_rows // 8, 8), (desc(heads=32), 8192 * 32, 32)):
        assert I.ios_attn_tree_work_bytes(d, n, most) > 0


# ---------------------------------------------------------------- the check of drafts

def test_verify():
    size = I.ios_verify_work_bytes(check())
    ok = dict(d=check(), p=rows(), q=rows(), tokens=P, parent=P, cu=P, accept=P, sample=P, path=P, count=P, next=P,
              work=P, size=size)

    def call(**kw):
        a = {**ok, **kw}
        I.ios_verify(a["d"], a["p"], a["q"], a["tokens"], a["parent"], a["cu"], a["accept"], a["sample"], a["path"],
                     a["count"], a["next"], a["work"], a["size"])
    for kw in (dict(dtype=3), dict(dtype=-1), dict(seqs=0), dict(seqs=65536), dict(vocab=0), dict(vocab=-5),
               dict(max_drafts=0), dict(max_drafts=65)):
        refused("IOS_E_ARG", lambda kw=kw: call(d=check(**kw)))
        refused("IOS_E_ARG", I.ios_verify_work_bytes, check(**kw))
    refused("IOS_E_ARG", lambda: call(p=None))
    for t in ("p", "q"):
        refused("IOS_E_ARG", lambda t=t: call(**{t: rows(data=0)}))
        refused("IOS_E_ARG", lambda t=t: call(**{t: rows(data=P + 2)}))
        refused("IOS_E_ARG", lambda t=t: call(**{t: rows(stride=-1)}))
        refused("IOS_E_ARG", lambda t=t: call(**{t: rows(n=-1)}))
        refused("IOS_E_SHAPE", lambda t=t: call(**{t: rows(n=11)}))
    for name in ("tokens", "parent", "cu", "accept", "sample", "path", "count", "next"):
        refused("IOS_E_ARG", lambda name=name: call(**{name: 0}))
    big = check(vocab=1 << 20, seqs=1)
    need = I.ios_verify_work_bytes(big)
    if need:
        refused("IOS_E_ARG", lambda: call(d=big, work=P, size=need - 1))
        refused("IOS_E_ARG", lambda: call(d=big, work=P + 4, size=need))
        refused("IOS_E_ARG", lambda: call(d=big, work=0, size=0))
