"""The decoder operators on the GPU against plain implementations in 64 bits:
prompt attention, the 4-bit cache (bit for bit), single-token attention over
it, and its pages (against a model that keeps pages in Python lists).

Tolerances are bounds, element by element.  With u the relative rounding error
of the output's type, A_i = sum_j softmax_j |v_j| and the scores computed in 32
bits (error at most g = 2^-23 (head_dim + 8) scale max_j sum_d |q_d k_d|):

    |o - ref| <= u |ref| + A (w + 2 g + 2^-24 (keys + 256))

where w is what the operator rounds before its second product: p to the type
for 16-bit prompts (u), p and the held value to f16 for the cache with bf16
results (2^-10; below f16's normal range 2^-25 each), p times the scale to 16
bits for f16 results (2^-16) and to 24 for float32 (2^-23), in both cases with
codes up to 143 in the place of values of a group (at most 16 times as large),
nothing for float32 prompts."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
I = pytest.importorskip("paper_2011_01302_amd")

DEV = "cuda:0"
TYPES = {"f32": (torch.float32, I.IOS_F32, 2.0 ** -24), "f16": (torch.float16, I.IOS_F16, 2.0 ** -11),
         "bf16": (torch.bfloat16, I.IOS_BF16, 2.0 ** -8)}


def stream():
    return torch.cuda.current_stream().cuda_stream


def toks(t):
    return I.ios_tokens(t.data_ptr(), t.shape[0], t.stride(0), t.stride(1))


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def offsets(lens):
    return [0] + [int(x) for x in np.cumsum(lens)]


def randn(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(DEV)


def desc(typ, heads, kv, dim, seqs, causal=0, max_keys=0, scale=None):
    d = I.ios_attn_desc()
    d.dtype, d.heads, d.kv_heads, d.head_dim, d.seqs = TYPES[typ][1], heads, kv, dim, seqs
    d.causal, d.max_keys, d.scale = causal, max_keys, 1 / math.sqrt(dim) if scale is None else scale
    return d


def attend(q, k, v, scale, seen):
    """64-bit attention of rows q [n][d] over k, v [m][d]; seen [n][m].  Unseen values take no part, whatever they
    are.  Returns the output, A, the log-sum-exp and the bound g."""
    q, k, v = (x.double().cpu() for x in (q, k, v))
    n, m = q.shape[0], k.shape[0]
    out, a = torch.zeros(n, v.shape[1], dtype=torch.float64), torch.zeros(n, v.shape[1], dtype=torch.float64)
    lse, g = torch.full((n,), -math.inf, dtype=torch.float64), torch.zeros(n, 1, dtype=torch.float64)
    if m == 0 or n == 0:
        return out, a, lse, g
    s = torch.where(seen, (q @ k.nan_to_num(0.0, 0.0, 0.0).T) * scale, -math.inf)
    rows = seen.any(1)
    lse[rows] = torch.logsumexp(s[rows], 1)
    p = torch.zeros_like(s)
    p[rows] = torch.exp(s[rows] - lse[rows, None])
    fin = torch.isfinite(v)
    v0 = torch.where(fin, v, 0.0)
    out, a = p @ v0, p @ v0.abs()
    if not fin.all():
        see = seen.double()
        nan, up, dn = (see @ x.double() > 0 for x in (torch.isnan(v), v == math.inf, v == -math.inf))
        out = torch.where(up, math.inf, torch.where(dn, -math.inf, out))
        out = torch.where(nan | (up & dn), math.nan, out)
    g = 2.0 ** -23 * (q.shape[1] + 8) * abs(scale) * torch.where(
        seen, q.abs() @ k.nan_to_num(0.0, 0.0, 0.0).abs().T, 0.0).amax(1, keepdim=True)
    return out, a, lse, g


def check(got, ref, a, g, u, w, keys, extra=0.0, what=""):
    got = got.double().cpu()
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))
    bound = u * ref.abs() + a * (w + 2 * g + 2.0 ** -24 * (keys + 256)) + extra + 2.0 ** -40
    ok = same | ((got - ref).abs() <= bound)
    assert ok.all(), (what, int((~ok).sum()), float(((got - ref).abs() / bound)[~ok].max()))


def causal_mask(lq, lk, causal):
    m = torch.ones(lq, lk, dtype=torch.bool)
    return m.tril(lk - lq) if causal else m


def prompt(typ, q, k, v, lq, lk, causal, scale=None, work=True):
    heads, kv, dim = q.shape[1], k.shape[1], q.shape[2]
    d = desc(typ, heads, kv, dim, len(lq), causal, max(lk + [0]), scale)
    out = torch.full_like(q, 7.0)
    out = torch.empty(q.shape, dtype=q.dtype, device=DEV).fill_(7.0)
    lse = torch.full((heads, q.shape[0]), 7.0, device=DEV)
    n = I.ios_attn_work_bytes(d, q.shape[0]) if work else 0
    w = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV)
    cq, ck = i32(offsets(lq)), i32(offsets(lk))
    I.ios_attn_prompt(d, toks(q), toks(k), toks(v), toks(out), lse.data_ptr(), cq.data_ptr(), ck.data_ptr(),
                      w.data_ptr() if n else 0, n, stream())
    torch.cuda.synchronize()
    return out, lse, d.scale


def check_prompt(typ, q, k, v, lq, lk, causal, scale=None, what="", work=True):
    print("\n[gpu-case] prompt", typ, tuple(q.shape), k.shape[1], lq, lk, causal, what, flush=True)
    out, lse, scale = prompt(typ, q, k, v, lq, lk, causal, scale, work)
    u = TYPES[typ][2]
    oq, ok = offsets(lq), offsets(lk)
    ratio = q.shape[1] // k.shape[1]
    for i in range(len(lq)):
        for h in range(q.shape[1]):
            ref, a, l64, g = attend(q[oq[i]:oq[i + 1], h], k[ok[i]:ok[i + 1], h // ratio],
                                    v[ok[i]:ok[i + 1], h // ratio], scale, causal_mask(lq[i], lk[i], causal))
            check(out[oq[i]:oq[i + 1], h], ref, a, g, u, 0.0 if typ == "f32" else u, lk[i], what=(what, i, h))
            got = lse[h, oq[i]:oq[i + 1]].double().cpu()
            fin = torch.isfinite(l64)
            assert torch.equal(got[~fin], l64[~fin])
            err = (got - l64).abs()[fin]
            assert (err <= (2 * g[fin, 0] + 2.0 ** -22 * (1 + l64[fin].abs()) + 2.0 ** -24 * (lk[i] + 256))).all()
    if oq[-1] < q.shape[0]:
        assert (out[oq[-1]:] == 7).all() and (lse[:, oq[-1]:] == 7).all()     # rows of no sequence
    return out


PROMPTS = [
    ([1], [1], 1), ([0, 5, 0], [3, 5, 0], 1), ([64, 63, 65], [64, 63, 65], 1), ([127, 129, 128], [127, 129, 128], 1),
    ([33, 1, 200], [333, 777, 200], 1), ([70, 300], [40, 0], 1), ([70, 300], [40, 0], 0), ([1, 31, 2], [64, 65, 700], 0),
    ([511], [513], 1),
]


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompt_lengths(typ, case):
    lq, lk, causal = PROMPTS[case]
    dt = TYPES[typ][0]
    q = randn((sum(lq) + 3, 6, 64), dt, case)
    k, v = randn((sum(lk) + 2, 2, 64), dt, case + 50), randn((sum(lk) + 2, 2, 64), dt, case + 90)
    k[sum(lk):], v[sum(lk):] = math.nan, math.nan          # rows of no sequence, seen by nobody
    check_prompt(typ, q, k, v, lq, lk, causal)


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 24, 32, 40, 56, 72, 96, 104, 120, 128])
def test_prompt_head_dims(typ, dim):
    dt = TYPES[typ][0]
    lq, lk = [130, 17], [190, 17]
    check_prompt(typ, randn((147, 2, dim), dt, 1), randn((207, 1, dim), dt, 2), randn((207, 1, dim), dt, 3), lq, lk, 1)


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
def test_prompt_strides(typ):
    """Heads before tokens, slices of a joint projection, one value row for all tokens, one head for all heads."""
    dt, n = TYPES[typ][0], 150
    joint = randn((n, 4 + 2 + 2, 48), dt, 4)
    q, k, v = joint[:, :4], joint[:, 4:6], joint[:, 6:]
    check_prompt(typ, q, k, v, [n], [n], 1, what="joint")
    qh, kh = randn((4, n, 48), dt, 5).transpose(0, 1), randn((2, n, 48), dt, 6).transpose(0, 1)
    check_prompt(typ, qh, kh, v, [n], [n], 0, what="heads first")
    check_prompt(typ, q, k, v[:1].expand(n, 2, 48), [n], [n], 1, what="one value")
    check_prompt(typ, q, k[:, :1].expand(n, 2, 48), v, [n], [n], 1, what="one key head")


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
def test_prompt_hidden_infinities_and_nan(typ):
    """A key or value that a row does not see never changes the row; those that it sees do as in the definition."""
    dt, n = TYPES[typ][0], 300
    q, k, v = randn((n, 2, 64), dt, 7), randn((n, 1, 64), dt, 8), randn((n, 1, 64), dt, 9)
    v[90, 0, 3], v[130, 0, 5], v[131, 0, 6], v[131, 0, 5] = math.nan, math.inf, -math.inf, -math.inf
    v[299] = math.inf
    check_prompt(typ, q, k, v, [n], [n], 1, what="values")
    k2 = k.clone()
    k2[200] = math.nan
    out, lse, _ = prompt(typ, q, k2, randn((n, 1, 64), dt, 9), [n], [n], 1)
    ref, lse0, _ = prompt(typ, q, k, randn((n, 1, 64), dt, 9), [n], [n], 1)
    assert torch.equal(out[:200], ref[:200]) and torch.equal(lse[:, :200], lse0[:, :200])
    assert torch.isnan(out[200:]).all()
    # the lowest and largest values of the type, hidden
    big = torch.finfo(dt).max
    k3, v3 = k.clone(), randn((n, 1, 64), dt, 9)
    k3[250:], v3[250:] = -big, big
    got, _, _ = prompt(typ, q, k3, v3, [n], [n], 1)
    assert torch.equal(got[:250], ref[:250])


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.125, 0.0, 1.0, 2.0 ** -20])
def test_prompt_scales(typ, scale):
    dt, n = TYPES[typ][0], 200
    check_prompt(typ, randn((n, 2, 64), dt, 1), randn((n, 2, 64), dt, 2), randn((n, 2, 64), dt, 3), [n], [n], 1, scale)


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
def test_prompt_growing_scores(typ):
    """Keys sorted by their score, so that the running maximum grows all the way, in both directions."""
    dt, n = TYPES[typ][0], 700
    q = torch.ones(n, 1, 32).to(dt).to(DEV)
    up = torch.linspace(-4, 4, n)[:, None, None].expand(n, 1, 32).to(dt).to(DEV).contiguous()
    v = randn((n, 1, 32), dt, 3)
    check_prompt(typ, q, up, v, [n], [n], 0, 1.0)
    check_prompt(typ, q, up.flip(0).contiguous(), v, [n], [n], 0, 1.0)


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
def test_prompt_few_rows_many_keys(typ):
    """With a workspace the keys of few rows are spread over workgroups; the result agrees with and without."""
    dt = TYPES[typ][0]
    lq, lk = [1, 40, 3], [5000, 3000, 0]
    q, k, v = randn((50, 4, 64), dt, 1), randn((8000, 2, 64), dt, 2), randn((8000, 2, 64), dt, 3)
    check_prompt(typ, q, k, v, lq, lk, 1)
    check_prompt(typ, q, k, v, lq, lk, 1, work=False)


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 200])
def test_prompt_long_tail(typ, rows):
    """One key far ahead of 6000 equal ones, whose weights (2^-16.6) sum to 0.06."""
    dt, n = TYPES[typ][0], 6000
    q = torch.zeros(rows, 1, 32, dtype=dt, device=DEV)
    q[:, :, 0] = 1.0
    k, v = torch.zeros(n, 1, 32, dtype=dt, device=DEV), torch.ones(n, 1, 32, dtype=dt, device=DEV)
    k[77, 0, 0], v[77] = 11.5, -1.0
    check_prompt(typ, q, k, v, [rows], [n], 0, 1.0)


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("lead", [11.5, 18.0])
def test_decode_long_tail(typ, lead):
    """As above over the cache; with a lead of 18 each of the others weighs 2^-26."""
    n = 50000 if lead > 12 else 6000
    c = Cache(1, 32, 256, 200, 1, 200)
    c.place([n])
    k, v = torch.zeros(n, 1, 32, device=DEV), torch.ones(n, 1, 32, device=DEV)
    k[77, 0, 0], v[77] = lead, -1.0
    c.append(k, v, [0], [n], "f32")
    q = torch.zeros(1, 1, 32, dtype=TYPES[typ][0], device=DEV)
    q[:, :, 0] = 1.0
    check_decode(typ, c, q, [0], [held(k)], [held(v)], [n], max_keys=n, scale=1.0)


def test_prompt_many_sequences():
    """More sequences than lanes search at once."""
    lens = [(7 * i) % 5 for i in range(300)]
    n = sum(lens)
    q, k, v = (randn((n, 1, 32), torch.float16, s) for s in (1, 2, 3))
    out, _, scale = prompt("f16", q, k, v, lens, lens, 1)
    o = offsets(lens)
    for i, m in enumerate(lens):
        ref, a, _, g = attend(q[o[i]:o[i] + m, 0], k[o[i]:o[i] + m, 0], v[o[i]:o[i] + m, 0], scale, causal_mask(m, m, 1))
        check(out[o[i]:o[i] + m, 0], ref, a, g, 2.0 ** -11, 2.0 ** -11, m)


@pytest.mark.parametrize("typ", ["f16", "f32"])
@pytest.mark.parametrize("n", [3, 100])
def test_prompt_offsets_that_start_later(typ, n):
    """The first sequence begins behind rows that belong to none."""
    dt, lens, skip = TYPES[typ][0], [1 + 3 * (i % 7) for i in range(n)], 300
    total = skip + sum(lens)
    q, k, v = (randn((total, 2, 32), dt, s) for s in (1, 2, 3))
    d = desc(typ, 2, 2, 32, n, 1, 32)
    out = torch.full_like(q, 7.0)
    o = [skip + x for x in offsets(lens)]
    cu = i32(o)
    I.ios_attn_prompt(d, toks(q), toks(k), toks(v), toks(out), 0, cu.data_ptr(), cu.data_ptr(), 0, 0, stream())
    torch.cuda.synchronize()
    assert (out[:skip] == 7).all()
    for i in range(0, n, 7):
        ref, a, _, g = attend(q[o[i]:o[i + 1], 1], k[o[i]:o[i + 1], 1], v[o[i]:o[i + 1], 1], d.scale,
                              causal_mask(lens[i], lens[i], 1))
        u = TYPES[typ][2]
        check(out[o[i]:o[i + 1], 1], ref, a, g, u, 0.0 if typ == "f32" else u, lens[i])


def test_prompt_bad_offsets_stay_inside():
    """Offsets that leave the tensors or descend are clipped: no fault, and sound sequences keep their results."""
    q, k, v = (randn((200, 2, 64), torch.float16, s) for s in (1, 2, 3))
    d = desc("f16", 2, 2, 64, 3, 1)
    out = torch.empty_like(q)
    cu = i32([0, 100, 1000000, -5])
    I.ios_attn_prompt(d, toks(q), toks(k), toks(v), toks(out), 0, cu.data_ptr(), cu.data_ptr(), 0, 0, stream())
    torch.cuda.synchronize()
    ref, a, _, g = attend(q[:100, 0], k[:100, 0], v[:100, 0], d.scale, causal_mask(100, 100, 1))
    check(out[:100, 0], ref, a, g, 2.0 ** -11, 2.0 ** -11, 100)


def test_prompt_graph_and_stream():
    """Recorded on a stream of its own, replayed on other lengths and values with eager work between."""
    q, k, v = (randn((256, 4, 64), torch.bfloat16, s) for s in (1, 2, 3))
    out, cu = torch.zeros_like(q), i32([0, 100, 256])
    d = desc("bf16", 4, 4, 64, 2, 1, 256)
    call = lambda: I.ios_attn_prompt(d, toks(q), toks(k), toks(v), toks(out), 0, cu.data_ptr(), cu.data_ptr(), 0, 0,
                                     stream())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for cut in (100, 7, 255, 100):
        cu.copy_(i32([0, cut, 256]))
        q.copy_(randn(q.shape, q.dtype, cut))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and out.abs().sum() > 0


# ---------------------------------------------------------------- the cache

class Cache:
    """A cache's tensors.  The pool is filled with NaN patterns: nothing may depend on what it held."""

    def __init__(self, kv, dim, page, pages, slots, row, layers=1, fill=0xFE):
        c = I.ios_cache()
        c.layers, c.kv_heads, c.head_dim, c.page_tokens, c.pages, c.slots, c.row = layers, kv, dim, page, pages, slots, row
        self.c = c
        self.pool = torch.full((layers, pages, I.ios_cache_page_bytes(c)), fill, dtype=torch.uint8, device=DEV)
        self.refs, self.lens = torch.zeros(pages, dtype=torch.int32, device=DEV), torch.zeros(slots, dtype=torch.int32, device=DEV)
        self.table = torch.full((slots, row), -1, dtype=torch.int32, device=DEV)
        self.work = torch.zeros(I.ios_cache_work_bytes(c), dtype=torch.uint8, device=DEV)
        c.pool, c.refs, c.table, c.lens, c.work = (t.data_ptr() for t in
                                                   (self.pool, self.refs, self.table, self.lens, self.work))

    def place(self, lens, seed=0):
        """Sequences of these lengths on shuffled pages."""
        t = self.c.page_tokens
        order = torch.randperm(self.c.pages, generator=torch.Generator().manual_seed(seed)).tolist()
        at = 0
        for i, m in enumerate(lens):
            n = -(-m // t)
            self.table[i, :n] = i32(order[at:at + n])
            self.refs[i32(order[at:at + n]).long()] = 1
            self.lens[i] = m
            at += n

    def reserve(self, seqs, add):
        a, b = i32(seqs), i32(add)
        I.ios_cache_reserve(self.c, len(seqs), a.data_ptr(), b.data_ptr(), stream())
        torch.cuda.synchronize()

    def append(self, k, v, seqs, lens, typ, layer=0):
        a, b = i32(seqs), i32(offsets(lens))
        I.ios_cache_append(self.c, layer, TYPES[typ][1], toks(k), toks(v), len(seqs), a.data_ptr(), b.data_ptr(), stream())
        torch.cuda.synchronize()

    def read(self, seqs, lens, typ="f32", layer=0):
        shape = (sum(lens), self.c.kv_heads, self.c.head_dim)
        k, v = (torch.full(shape, 9.0, dtype=TYPES[typ][0], device=DEV) for _ in range(2))
        a, b = i32(seqs), i32(offsets(lens))
        I.ios_cache_read(self.c, layer, TYPES[typ][1], toks(k), toks(v), len(seqs), a.data_ptr(), b.data_ptr(), stream())
        torch.cuda.synchronize()
        return k, v


def held(x):
    """What the cache holds for x, from the format's definition, in numpy's float32."""
    x = x.float().cpu().numpy()
    y = np.minimum(np.maximum(x, np.float32(-61440)), np.float32(61440)).reshape(x.shape[:-1] + (-1, 32))
    lo, hi = y.min(-1, keepdims=True), y.max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        z = lo.astype(np.float16).astype(np.float32)
        s = ((hi - lo) * np.float32(1.0 / 15.0)).astype(np.float16).astype(np.float32)
        c = np.where(s > 0, np.clip(np.rint((y - z) / s), 0, 15), 0).astype(np.float32)
        out = z + s * c
    out[np.isnan(y).any(-1)] = np.nan
    return torch.from_numpy(out.reshape(x.shape))


def equal(a, b):
    a, b = a.cpu(), b.cpu()
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim,page", [(32, 32), (64, 256), (96, 64), (128, 128)])
def test_cache_holds_the_formats_values(typ, dim, page):
    print("\n[gpu-case] cache", typ, dim, page, flush=True)
    dt, lens = TYPES[typ][0], [1, 31, 0, 32, 33, 300]
    c = Cache(3, dim, page, 40, 8, 12)
    c.place(lens)
    k, v = (randn((sum(lens), 3, dim), dt, s, 3.0) for s in (1, 2))
    k[:, 1] += 40.0                              # an offset, a constant group, tiny and huge values
    k[3, 0, :32], v[5, 2, :32] = 2.5, 0.0
    v[:, 1] *= 1e-6
    k[7, 2] *= 1e4 if typ != "f16" else 1e3
    v[9, 0, 1], v[9, 0, 2], k[11, 1, 31], v[40, 2, 5] = math.inf, -math.inf, -math.inf, math.nan
    c.append(k, v, list(range(6)), lens, typ)
    gk, gv = c.read(list(range(6)), lens)
    assert equal(gk, held(k)) and equal(gv, held(v))
    assert not torch.isnan(gk).any()
    bk, bv = c.read(list(range(6)), lens, "bf16")
    assert equal(bk.float(), held(k).to(torch.bfloat16).float()) and equal(bv.float(), held(v).to(torch.bfloat16).float())
    hk, hv = c.read(list(range(6)), lens, "f16")
    assert torch.isfinite(hk).all() and equal(hk.float(), held(k).to(torch.float16).float())


@pytest.mark.parametrize("dim,page", [(32, 64), (96, 32), (128, 64)])
def test_cache_grows_in_pieces(dim, page):
    """Pieces of every length, single tokens among them, leave what was there as it was."""
    c = Cache(2, dim, page, 64, 3, 20)
    rng, all_k, all_v = np.random.default_rng(5), [[], [], []], [[], [], []]
    for step in range(12):
        seqs = [2, 0] if step % 3 else [1, 2, 0]
        lens = [1] * len(seqs) if step % 2 else [int(x) for x in rng.integers(0, 70, len(seqs))]
        k, v = (randn((sum(lens) + 1, 2, dim), torch.float16, 10 * step + s) for s in (1, 2))
        c.reserve(seqs, lens)
        c.append(k, v, seqs, lens, "f16")
        o = offsets(lens)
        for i, s in enumerate(seqs):
            all_k[s].append(k[o[i]:o[i + 1]])
            all_v[s].append(v[o[i]:o[i + 1]])
    assert I.ios_cache_status(c.c, stream()) == 0
    lens = [sum(x.shape[0] for x in all_k[s]) for s in range(3)]
    assert c.lens.tolist() == lens
    gk, gv = c.read([0, 1, 2], lens)
    assert equal(gk, held(torch.cat([torch.cat(x) for x in all_k])))
    assert equal(gv, held(torch.cat([torch.cat(x) for x in all_v])))


def test_cache_append_and_read_edges():
    """Slots out of range, more tokens than the sequence has, a missing page."""
    c = Cache(1, 64, 32, 8, 4, 4)
    c.place([40, 5])
    k, v = randn((60, 1, 64), torch.float32, 1), randn((60, 1, 64), torch.float32, 2)
    c.append(k, v, [0, 1, -1, 99], [45, 5, 5, 5], "f32")
    gk, gv = c.read([0, 1, -1, 99], [45, 5, 5, 5])
    assert equal(gk[5:50], held(k[5:50])) and equal(gv[5:50], held(v[5:50]))
    assert (gk[:5] == 0).all() and (gk[50:] == 0).all() and (gv[:5] == 0).all() and (gv[50:] == 0).all()
    c.table[0, 1] = 12345                        # no such page: reads as 0, writes nowhere
    before = c.pool.clone()
    c.append(k[:8], v[:8], [0], [8], "f32")
    assert torch.equal(before, c.pool)
    gk, _ = c.read([0], [40])
    assert equal(gk[:32], held(k[5:37])) and (gk[32:] == 0).all()


def test_cache_offsets_that_start_later_or_descend():
    c = Cache(1, 32, 32, 16, 3, 4)
    c.place([70, 40, 33])
    k, v = randn((400, 1, 32), torch.float32, 1), randn((400, 1, 32), torch.float32, 2)
    seqs, cu = i32([0, 1]), i32([200, 270, 310])
    I.ios_cache_append(c.c, 0, I.IOS_F32, toks(k), toks(v), 2, seqs.data_ptr(), cu.data_ptr(), stream())
    gk, gv = c.read([0, 1], [70, 40])
    assert equal(gk, held(k[200:310])) and equal(gv, held(v[200:310]))
    out = torch.full_like(k, 9.0)
    I.ios_cache_read(c.c, 0, I.IOS_F32, toks(out), toks(out.clone()), 2, seqs.data_ptr(), cu.data_ptr(), stream())
    torch.cuda.synchronize()
    assert (out[:200] == 9).all() and equal(out[200:310], held(k[200:310])) and (out[310:] == 9).all()
    before = c.pool.clone()
    for bad in ([390, 100, 50], [10 ** 9, -5, -9], [400, 400, 0]):
        cu = i32(bad)
        I.ios_cache_append(c.c, 0, I.IOS_F32, toks(k), toks(v), 2, seqs.data_ptr(), cu.data_ptr(), stream())
    torch.cuda.synchronize()
    assert torch.equal(before, c.pool)


def test_cache_append_strides():
    c = Cache(2, 64, 32, 8, 2, 8)
    c.place([50, 20])
    joint = randn((70, 2, 2, 64), torch.bfloat16, 3)
    c.append(joint[:, 0], joint[:, 1], [0, 1], [50, 20], "bf16")
    gk, gv = c.read([0, 1], [50, 20])
    assert equal(gk, held(joint[:, 0])) and equal(gv, held(joint[:, 1]))


def decode(c, typ, q, seqs, max_keys=0, work=True, layer=0, scale=None):
    d = desc(typ, q.shape[1], c.c.kv_heads, c.c.head_dim, len(seqs), 0, max_keys, scale)
    n = I.ios_attn_work_bytes(d, len(seqs)) if work else 0
    w = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV)
    out, lse, s = torch.empty_like(q), torch.full((q.shape[1], len(seqs)), 7.0, device=DEV), i32(seqs)
    I.ios_attn_cache(c.c, layer, d, toks(q), toks(out), lse.data_ptr(), s.data_ptr(), w.data_ptr() if n else 0, n, stream())
    torch.cuda.synchronize()
    return out, lse, d.scale


def decode_rounding(typ, v, n):
    """w, keys and the absolute part of the bound for single-token attention over values v [n][d]."""
    if typ == "bf16":
        return 2.0 ** -10 + 2.0 ** -21, n, 2.0 ** -25 * (float(v.double().abs().sum(0).max()) + 1)
    # what a group's codes, scales and zero points sum to in 32 bits: up to 32 times its largest value
    big = 32 * float(v.double().abs().max())
    return 0.0, n, (2.0 ** -16 if typ == "f16" else 2.0 ** -23) * big / 2 + 2.0 ** -24 * (n + 256) * big


def check_decode(typ, c, q, seqs, k, v, lens, **kw):
    """k, v: the values held, one tensor per slot."""
    out, lse, scale = decode(c, typ, q, seqs, **kw)
    u, ratio = TYPES[typ][2], q.shape[1] // c.c.kv_heads
    for i, s in enumerate(seqs):
        for h in range(q.shape[1]):
            n = lens[s] if 0 <= s < len(lens) else 0
            if n == 0:
                assert (out[i, h] == 0).all() and lse[h, i] == -math.inf
                continue
            kk, vv = k[s][:, h // ratio], v[s][:, h // ratio]
            ref, a, l64, g = attend(q[i:i + 1, h], kk, vv, scale, torch.ones(1, n, dtype=torch.bool))
            check(out[i:i + 1, h], ref, a, g, u, *decode_rounding(typ, vv, n), (i, h))
            assert abs(float(lse[h, i]) - float(l64)) <= float(2 * g) + 2.0 ** -22 * (1 + abs(float(l64))) + 2.0 ** -24 * (n + 256)


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim,page,kv,ratio", [(32, 32, 2, 1), (64, 64, 1, 8), (96, 32, 2, 5), (128, 128, 2, 4),
                                               (128, 32, 1, 16), (64, 256, 1, 17), (32, 64, 1, 40)])
def test_decode(typ, dim, page, kv, ratio):
    print("\n[gpu-case] decode", typ, dim, page, kv, ratio, flush=True)
    lens = [0, 1, 31, 32, 33, 64, 127, 1000]
    c = Cache(kv, dim, page, 64, 10, 40)
    c.place(lens, 3)
    k, v = randn((sum(lens), kv, dim), torch.float32, 1), randn((sum(lens), kv, dim), torch.float32, 2, 5.0)
    c.append(k, v, list(range(len(lens))), lens, "f32")
    o = offsets(lens)
    hk, hv = ([x[o[i]:o[i + 1]] for i in range(len(lens))] for x in (held(k), held(v)))
    seqs = [7, 0, 1, 2, -1, 3, 4, 5, 6, 9, 12345]
    q = randn((len(seqs), kv * ratio, dim), TYPES[typ][0], 3)
    q[2] *= 30.0                                 # one key far ahead of the others
    q[3] *= 2.0 ** -12
    q[5, 0] = 0.0
    for kw in (dict(), dict(work=False), dict(max_keys=1000)):
        check_decode(typ, c, q, seqs, hk, hv, lens, **kw)


@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
def test_decode_long_and_strided(typ):
    lens = [9000, 2049]
    c = Cache(2, 64, 64, 200, 2, 150)
    c.place(lens, 4)
    k, v = randn((sum(lens), 2, 64), torch.float16, 1), randn((sum(lens), 2, 64), torch.float16, 2)
    c.append(k, v, [0, 1], lens, "f16")
    o = offsets(lens)
    hk, hv = ([x[o[i]:o[i + 1]] for i in range(2)] for x in (held(k), held(v)))
    q = randn((6, 2, 64), TYPES[typ][0], 3).transpose(0, 1)          # heads first
    check_decode(typ, c, q, [1, 0], hk, hv, lens, max_keys=9000)
    check_decode(typ, c, q, [1, 0], hk, hv, lens, max_keys=100)      # a wrong bound only costs speed
    check_decode(typ, c, q, [0, 0], hk, hv, lens, scale=-0.3)


def test_decode_large_values_and_nan():
    """The ends of the format's range stay finite; a NaN group reaches the rows that read it."""
    c = Cache(1, 32, 32, 8, 2, 4)
    c.place([40, 40])
    k = randn((80, 1, 32), torch.float32, 1)
    v = torch.full((80, 1, 32), 60000.0, device=DEV)
    v[::2] = -60000.0
    v[:, :, ::3] *= -1e6
    v[50, 0, 4] = math.nan
    c.append(k, v, [0, 1], [40, 40], "f32")
    q = randn((2, 1, 32), torch.bfloat16, 2)
    out, _, _ = decode(c, "bf16", q, [0, 1])
    hk, hv = held(k), held(v)
    ref, a, _, g = attend(q[:1, 0], hk[:40, 0], hv[:40, 0], 1 / math.sqrt(32), torch.ones(1, 40, dtype=torch.bool))
    check(out[:1, 0], ref, a, g, 2.0 ** -8, 2.0 ** -10 + 2.0 ** -21, 40, 1e-3)
    assert torch.isnan(out[1]).all()


def test_decode_pool_beyond_32_bits():
    """A pool of more than 4 GiB: pages at its end, in the last layer."""
    c = Cache(8, 128, 256, 1700, 2, 8, layers=8)
    assert c.pool.numel() > 1 << 32
    lens = [300, 257]
    for i, pages in enumerate(([1699, 3], [1650, 1698])):
        c.table[i, :2] = i32(pages)
        c.refs[i32(pages).long()] = 1
        c.lens[i] = lens[i]
    k, v = randn((557, 8, 128), torch.bfloat16, 1), randn((557, 8, 128), torch.bfloat16, 2)
    c.append(k, v, [0, 1], lens, "bf16", layer=7)
    gk, gv = c.read([0, 1], lens, layer=7)
    assert equal(gk, held(k)) and equal(gv, held(v))
    q = randn((2, 8, 128), torch.bfloat16, 3)
    out, _, scale = decode(c, "bf16", q, [1, 0], layer=7)
    for i, rows in enumerate((slice(300, 557), slice(0, 300))):
        ref, a, _, g = attend(q[i:i + 1, 5], held(k)[rows, 5], held(v)[rows, 5], scale,
                              torch.ones(1, rows.stop - rows.start, dtype=torch.bool))
        check(out[i:i + 1, 5], ref, a, g, 2.0 ** -8, 2.0 ** -10, 300, 2.0 ** -15)


def test_decode_graph():
    """Recorded once; replayed while the sequences grow, eager work and synchronisation between."""
    c = Cache(1, 64, 32, 32, 2, 16)
    q, out, seqs = randn((2, 4, 64), torch.float16, 1), torch.zeros(2, 4, 64, dtype=torch.float16, device=DEV), i32([0, 1])
    k, v = randn((2, 1, 64), torch.float16, 2), randn((2, 1, 64), torch.float16, 3)
    add, cu, d = i32([1, 1]), i32([0, 1, 2]), desc("f16", 4, 1, 64, 2, 0, 512)
    n = I.ios_attn_work_bytes(d, 2)
    w = torch.zeros(max(n, 16), dtype=torch.uint8, device=DEV)

    def step():
        I.ios_cache_reserve(c.c, 2, seqs.data_ptr(), add.data_ptr(), stream())
        I.ios_cache_append(c.c, 0, I.IOS_F16, toks(k), toks(v), 2, seqs.data_ptr(), cu.data_ptr(), stream())
        I.ios_attn_cache(c.c, 0, d, toks(q), toks(out), 0, seqs.data_ptr(), w.data_ptr(), n, stream())
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    ks, vs = [held(k)], [held(v)]
    for i in range(70):
        k.copy_(randn(k.shape, k.dtype, 100 + i))
        v.copy_(randn(v.shape, v.dtype, 200 + i))
        q.copy_(randn(q.shape, q.dtype, 300 + i))
        g.replay()
        torch.cuda.synchronize()
        ks.append(held(k))
        vs.append(held(v))
        assert c.lens.tolist() == [i + 2] * 2
        for s in range(2):
            kk, vv = (torch.stack([x[s, 0] for x in xs]) for xs in (ks, vs))
            ref, a, _, gg = attend(q[s], kk, vv, d.scale, torch.ones(4, i + 2, dtype=torch.bool))
            check(out[s], ref, a, gg, 2.0 ** -11, *decode_rounding("f16", vv, i + 2), i)
    assert I.ios_cache_status(c.c, stream()) == 0


# ---------------------------------------------------------------- pages

class Model:
    """The pages' rules, one sequence after the other."""

    def __init__(self, c):
        self.t, self.row, self.pages = c.c.page_tokens, c.c.row, c.c.pages
        self.rows, self.lens = [[] for _ in range(c.c.slots)], [0] * c.c.slots
        self.refs, self.pool = [0] * self.pages, c.pool.clone()

    def reserve(self, seqs, add):
        live = [(s, a) for s, a in zip(seqs, add) if 0 <= s < len(self.lens) and a > 0]
        shared = {}
        for i, (s, _) in enumerate(live):
            if self.lens[s] % self.t and self.refs[self.rows[s][-1]] > 1:
                shared.setdefault(self.rows[s][-1], []).append(i)
        copy = {i for p, xs in shared.items() for i in xs if not (len(xs) == self.refs[p] and i == xs[-1])}
        need, over = [], 0
        for i, (s, a) in enumerate(live):
            n = -(-(self.lens[s] + a) // self.t)
            over |= n > self.row
            need.append(n - len(self.rows[s]) + (i in copy))
        free = [p for p in range(self.pages) if self.refs[p] == 0]
        if over:
            return 2
        if sum(need) > len(free):
            return 1
        drop = []
        for i, (s, a) in enumerate(live):
            if i in copy:
                p = free.pop(0)
                self.pool[:, p] = self.pool[:, self.rows[s][-1]]
                drop.append(self.rows[s][-1])
                self.rows[s][-1], self.refs[p] = p, 1
            while len(self.rows[s]) * self.t < self.lens[s] + a:
                p = free.pop(0)
                self.rows[s].append(p)
                self.refs[p] = 1
            self.lens[s] += a
        for p in drop:
            self.refs[p] -= 1
        return 0

    def fork(self, parents, children):
        flag = 0
        for p, ch in zip(parents, children):
            if self.lens[ch]:
                flag = 4
                continue
            self.rows[ch], self.lens[ch] = list(self.rows[p]), self.lens[p]
            for x in self.rows[ch]:
                self.refs[x] += 1
        return flag

    def free(self, seqs):
        for s in seqs:
            if not 0 <= s < len(self.lens):
                continue
            for x in self.rows[s]:
                self.refs[x] -= 1
            self.rows[s], self.lens[s] = [], 0

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        src = [p for p in range(live, self.pages) if self.refs[p]]
        dst = [p for p in range(live) if not self.refs[p]]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.pool[:, b] = self.pool[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[to.get(x, x) for x in r] for r in self.rows]
        return live

    def check(self, c):
        assert c.lens.tolist() == self.lens
        assert c.refs.tolist() == self.refs
        assert c.table.tolist() == [r + [-1] * (self.row - len(r)) for r in self.rows]
        assert torch.equal(c.pool, self.pool)


@pytest.mark.parametrize("page,pages,slots,row,layers,seed", [(32, 50, 12, 10, 2, 0), (64, 24, 9, 5, 1, 1),
                                                               (32, 1, 2, 2, 3, 2), (256, 3000, 1500, 4, 1, 3)])
def test_pages_against_the_model(page, pages, slots, row, layers, seed):
    print("\n[gpu-case] pages", page, pages, slots, flush=True)
    c = Cache(1, 32, page, pages, slots, row, layers)
    c.pool.copy_(torch.randint(0, 256, c.pool.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(seed)))
    m, rng, live = Model(c), np.random.default_rng(seed), torch.zeros(1, dtype=torch.int32, device=DEV)
    for step in range(60):
        op = rng.integers(0, 5)
        order = [int(x) for x in rng.permutation(slots)[:rng.integers(1, slots + 1)]]
        if op <= 1:
            add = [int(x) for x in rng.integers(-1, 2 * page if op else 3, len(order))]
            if step % 7 == 0:
                order[0] = -1
            c.reserve(order, add)
            assert I.ios_cache_status(c.c, stream()) & 3 in ({0: [0], 1: [1], 2: [2, 3]}[m.reserve(order, add)])
        elif op == 2 and len(order) > 1:
            h = len(order) // 2
            parents, children = [order[int(x)] for x in rng.integers(0, h, len(order) - h)], order[h:]
            a, b = i32(parents), i32(children)
            I.ios_cache_fork(c.c, len(children), a.data_ptr(), b.data_ptr(), stream())
            assert I.ios_cache_status(c.c, stream()) == m.fork(parents, children)
        elif op == 3:
            a = i32(order[:max(1, len(order) // 3)] + [-7])[:slots]
            I.ios_cache_free(c.c, a.shape[0], a.data_ptr(), stream())
            m.free(a.tolist())
        else:
            I.ios_cache_compact(c.c, live.data_ptr(), stream())
            assert int(live) == m.compact()
        torch.cuda.synchronize()
        m.check(c)


def test_pages_all_sharers_reserve_at_once():
    """Three sharers of a partly filled page: two copies are made, the last one keeps the page."""
    c = Cache(1, 32, 32, 8, 4, 4)
    m = Model(c)
    for args in (([0], [40]),):
        c.reserve(*args)
        m.reserve(*args)
    a, b = i32([0, 0]), i32([1, 2])
    I.ios_cache_fork(c.c, 2, a.data_ptr(), b.data_ptr(), stream())
    m.fork([0, 0], [1, 2])
    c.reserve([1, 0, 2], [1, 1, 1])
    m.reserve([1, 0, 2], [1, 1, 1])
    m.check(c)
    assert c.refs.tolist() == [3, 1, 1, 1, 0, 0, 0, 0] and c.table[2, 1] == 1


def test_pages_copy_and_freed_twice():
    c = Cache(2, 64, 32, 10, 3, 4, layers=3)
    c.pool.copy_(torch.randint(0, 256, c.pool.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(1)))
    ref = c.pool.clone()
    src, dst = i32([1, 9, -1, 3]), i32([5, 0, 2, 10])
    I.ios_cache_copy(c.c, 4, src.data_ptr(), dst.data_ptr(), stream())
    torch.cuda.synchronize()
    ref[:, 5], ref[:, 0] = ref[:, 1].clone(), ref[:, 9].clone()
    assert torch.equal(c.pool, ref)
    c.reserve([0, 1], [50, 10])
    s = i32([0, 0, 1])
    I.ios_cache_free(c.c, 3, s.data_ptr(), stream())
    torch.cuda.synchronize()
    assert (c.refs == 0).all() and (c.lens == 0).all() and (c.table == -1).all()


def test_forked_sequences_keep_their_tokens():
    """Answers that share a prompt and then go their own ways read back what each of them wrote."""
    c = Cache(1, 64, 32, 40, 5, 8, layers=2)
    k, v = randn((45, 1, 64), torch.bfloat16, 1), randn((45, 1, 64), torch.bfloat16, 2)
    c.reserve([0], [45])
    for layer in range(2):
        c.append(k, v, [0], [45], "bf16", layer)
    a, b = i32([0, 0, 0]), i32([1, 2, 3])
    I.ios_cache_fork(c.c, 3, a.data_ptr(), b.data_ptr(), stream())
    new = []
    for step in range(3):
        c.reserve([0, 1, 2, 3], [1] * 4)
        x = randn((4, 1, 64), torch.bfloat16, 10 + step)
        for layer in range(2):
            c.append(x, x, [0, 1, 2, 3], [1] * 4, "bf16", layer)
        new.append(x)
        if step == 1:
            I.ios_cache_free(c.c, 1, i32([2]).data_ptr(), stream())
            I.ios_cache_compact(c.c, 0, stream())
    for layer in range(2):
        for s in (0, 1, 3):
            gk, gv = c.read([s], [48], layer=layer)
            tail = torch.cat([x[s:s + 1] for x in new])
            assert equal(gk, held(torch.cat([k, tail]))) and equal(gv, held(torch.cat([v, tail])))
        gk, _ = c.read([2], [1], layer=layer)
        assert equal(gk, held(new[2][2:3]))


def test_example_answers():
    """The example's path, end to end: answers differ, sharing holds, and the cache's prompt is what was written."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_maps.py")
    spec = importlib.util.spec_from_file_location("answer_maps", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    ids, pages, dec = ex.answers(3, 8)
    assert [len(r) for r in ids] == [8] * 3 and len({r[0] for r in ids}) == 3
    prompt, page = 1225, ex.PAGE
    own = -(-(prompt + 7) // page) - prompt // page          # pages that an answer does not share
    assert pages == [-(-prompt // page) + 3 * own, -(-prompt // page) + own]
    assert dec.lens.tolist() == [prompt, prompt + 7, 0, 0]
    assert sorted(set(dec.table[dec.table >= 0].tolist())) == list(range(pages[1]))
    assert ids == ex.answers(3, 8)[0]                        # the same again
