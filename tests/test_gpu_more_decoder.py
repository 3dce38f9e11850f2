"""Several tokens a step on the GPU, against plain implementations in 64 bits:
rotation by positions, rotated appends and kept drafts (bit for bit through the
cache), attention of drafted trees over the cache, and the check of the drafts.

Rotation.  The reference turns in 64 bits; cosine, sine, each product and the
sum are rounded to 24 bits and the result to the type (u, its half step):
    |a' - ref| <= u |ref| + 2^-22 amplitude (|a| + |b|) + 2^-25 2^-14.

Attention of drafts.  With p the softmax over cached keys z + s c and the drafts
that a row sees, A = sum p (|z| + 15 s) + sum p |v| and e the largest error of a
score, element by element:
    |o - ref| <= u |ref| + 2^-25 + (2 e + 2^-17) A + w + 2^-24 R (S + |ref|)
e   scale (2^-22 + 2^-24 (head_dim + 8)) sum_d |q_d| (|z| + 15 s) for cached keys
    (queries, their sums and middles z + 8 s in two 16-bit parts or more, 32-bit sums; for
    bf16 the values themselves may be rounded to f16, 2^-11 more), scale 2^-24 (head_dim + 10) sum |q k|
    for drafts, and 2^-17 for the exponential's argument (scores below 40) and value
w   roundings before the second product: for bf16 p and the value to f16 (2^-10 A); for f16
    both to two f16 parts, 2^-22 each, and the product of the second parts left out, 2^-22
    (2^-20 A); for both 2^-34 of the largest value a key for weights below f16's range; for
    float32 p s to three 16-bit parts times codes of up to 15; drafts' p to two parts of the
    type (2^-16 A)
S   what is summed in 32 bits: A
R   roundings one behind the other: 33 a tile for a quarter of the tiles at worst, 128
    for the drafts, 8 waves, 40 for rescaling and the last steps, and 128 for the parts (256
    at most, over two threads at least)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
I = pytest.importorskip("paper_2011_01302_amd")

from test_gpu_decoder import DEV, TYPES, Cache, desc, equal, held, i32, offsets, randn, stream, toks  # noqa: E402
from test_gpu_decoder_bounds import quantised  # noqa: E402

ALL = pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])


def rotary(dim, interleaved=0, amplitude=1.0, base=10000.0, *scaling):
    r = I.ios_rotary(dim, interleaved, amplitude)
    I.ios_rotary_freqs(r, base, *scaling)
    return r


def turned64(r, x, pos):
    """x [tokens][heads][dim] turned in 64 bits, and sum of a pair's absolute values."""
    x, n = x.double().cpu(), r.dim // 2
    f = torch.tensor(list(r.freq[:n]), dtype=torch.float64)
    z = torch.polar(torch.full((len(pos), n), 1.0, dtype=torch.float64), torch.tensor(pos, dtype=torch.float64)[:, None] * f)
    c, s = (r.amplitude * t[:, None] for t in (z.real, z.imag))
    at = torch.arange(n)
    ia, ib = (2 * at, 2 * at + 1) if r.interleaved else (at, at + n)
    a, b = x[..., ia], x[..., ib]
    out, size = x.clone(), torch.zeros_like(x)
    out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return out, size


def turned32(r, x, pos):
    """The same by the definition's own roundings, in numpy's float32."""
    n = r.dim // 2
    angle = np.array(pos, dtype=np.float64)[:, None] * np.array(r.freq[:n])
    c, s = ((np.float64(r.amplitude) * t).astype(np.float32)[:, None] for t in (np.cos(angle), np.sin(angle)))
    y = x.float().cpu().numpy()
    ia, ib = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if r.interleaved else (slice(0, n), slice(n, 2 * n))
    out = y.copy()
    out[..., ia], out[..., ib] = y[..., ia] * c - y[..., ib] * s, y[..., ia] * s + y[..., ib] * c
    return torch.from_numpy(out).to(x.dtype)


def rotate(typ, r, q, k, pos, qo=None, ko=None):
    dt = TYPES[typ][0]
    qo = torch.full(q.shape, 7.0, dtype=dt, device=DEV) if qo is None else qo
    ko = (torch.full(k.shape, 7.0, dtype=dt, device=DEV) if ko is None else ko) if k is not None else None
    p = i32(pos)
    I.ios_rotate(r, TYPES[typ][1], q.shape[2], toks(q), toks(qo), q.shape[1], toks(k) if k is not None else None,
                 toks(ko) if k is not None else None, k.shape[1] if k is not None else 0, p.data_ptr(), stream())
    torch.cuda.synchronize()
    return qo, ko


def check_turned(typ, r, x, pos, got):
    ref, size = turned64(r, x, pos)
    # (numbers of f16 below 2^-14 are 2^-24 apart, so half a step is 2^-25 there and not a share of the number)
    bound = TYPES[typ][2] * ref.abs() + 2.0 ** -22 * abs(r.amplitude) * size + (2.0 ** -25 if typ == "f16" else 2.0 ** -39)
    err = (got.double().cpu() - ref).abs()
    assert (err <= bound).all(), float((err / bound).max())
    step = turned32(r, x, pos)
    assert float((got.cpu() != step).float().mean()) <= 1e-3            # all but a few to the bit
    assert torch.equal(got[..., r.dim:], x[..., r.dim:])


# ---------------------------------------------------------------- rotation

@ALL
@pytest.mark.parametrize("inter", [0, 1])
@pytest.mark.parametrize("head,dim", [(8, 2), (8, 8), (40, 20), (64, 64), (64, 32), (80, 80), (96, 50), (128, 128),
                                      (128, 6), (120, 112)])
def test_rotate(typ, inter, head, dim):
    print("\n[gpu-case] rotate", typ, inter, head, dim, flush=True)
    n, dt = 37, TYPES[typ][0]
    q, k = randn((n, 5, head), dt, 1), randn((n, 2, head), dt, 2, 30.0)
    pos = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 131071, 10 ** 6] + [int(x) for x in np.random.default_rng(3).integers(0, 70000, n - 7)]
    r = rotary(dim, inter)
    qo, ko = rotate(typ, r, q, k, pos)
    check_turned(typ, r, q, pos, qo)
    check_turned(typ, r, k, pos, ko)
    # in place, and alone
    q2, k2 = q.clone(), k.clone()
    rotate(typ, r, q2, k2, pos, q2, k2)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    k3 = k.clone()
    rotate(typ, r, k3, None, pos, k3)
    assert torch.equal(k3, ko)


@pytest.mark.parametrize("heads,head,dim,inter,tokens", [(1, 8, 8, 1, 150001), (1, 128, 128, 0, 40000), (3, 40, 20, 0, 33333),
                                                         (300, 8, 2, 0, 1025)])
def test_rotate_many_tokens(heads, head, dim, inter, tokens):
    """As many tokens a workgroup as it takes, and heads in more than one turn of its threads."""
    r = rotary(dim, inter)
    q, pos = randn((tokens, heads, head), torch.float16, 1), [(7 * i) % 100003 for i in range(tokens)]
    got, _ = rotate("f16", r, q, None, pos)
    check_turned("f16", r, q, pos, got)


@ALL
def test_rotate_scaled_and_back(typ):
    dt, n = TYPES[typ][0], 2100                       # more than one workgroup's tokens
    q, k = randn((n, 3, 64), dt, 1), randn((n, 3, 64), dt, 2)
    pos = list(range(500000, 500000 + n))
    r = rotary(64, 0, 1.25, 500000.0, 8.0, 8192.0, 1.0, 4.0)
    qo, ko = rotate(typ, r, q, k, pos)
    check_turned(typ, r, q, pos, qo)
    check_turned(typ, r, k, pos, ko)
    for i in range(32):
        r.freq[i] = -r.freq[i]
    r.amplitude = 0.8
    back, _ = rotate(typ, r, qo, None, pos)
    # turned, rounded, turned back, rounded: u of each turned value, then the second call's own bound
    _, size = turned64(r, q, pos)
    u = TYPES[typ][2]
    assert ((back.double() - q.double()).abs().cpu() <= 1.25 * u * 2 * size + u * q.abs().double().cpu() + 2.0 ** -21 * size + 2.0 ** -20 * u).all()


@ALL
def test_rotate_gradient_is_the_rotation_back(typ):
    """<turn(x), y> = <x, turn back(y)>, and differences of a product with y along a direction."""
    n, pos = 5, [3, 70, 1000, 12345, 0]
    x, y = randn((n, 2, 32), torch.float32, 1), randn((n, 2, 32), torch.float32, 2)
    r = rotary(32, 1)
    tx, _ = rotate("f32", r, x, None, pos)
    for i in range(16):
        r.freq[i] = -r.freq[i]
    ty, _ = rotate("f32", r, y, None, pos)
    a, b = float((tx.double() * y.double()).sum()), float((x.double() * ty.double()).sum())
    size = float((x.double().abs() * y.double().abs().amax()).sum())
    assert abs(a - b) <= 2.0 ** -20 * size * 2


@ALL
@pytest.mark.parametrize("inter,dim,amplitude", [(0, 64, 1.0), (1, 40, 1.25), (0, 20, 0.75)])
def test_rotate_gradient_by_type_and_differences(typ, inter, dim, amplitude):
    """Of L(x) = <turn(x), y> the gradient is y turned with the frequencies negated: against differences of L along
    directions z.  x and z are eighths, so x + z and x - z are exact in every type, and L(x + z) - L(x - z) = 2 <z, gradient>
    but for each call's own roundings (as check_turned counts them), weighed by y and by 2 |z|."""
    n, dt = 9, TYPES[typ][0]
    pos = [0, 1, 3, 70, 1000, 12345, 100003, -5, 7]
    rng = np.random.default_rng(dim)
    eighths = lambda: torch.from_numpy(rng.integers(-16, 17, (n, 2, 64)) / 8.0).to(dt).to(DEV)  # noqa: E731
    x, y, r = eighths(), randn((n, 2, 64), dt, 2), rotary(dim, inter, amplitude)

    def bound(t):
        ref, size = turned64(r, t, pos)
        return TYPES[typ][2] * ref.abs() + 2.0 ** -22 * amplitude * size + (2.0 ** -25 if typ == "f16" else 2.0 ** -39)
    turned = {}
    zs = [eighths() for _ in range(4)]
    for i, z in enumerate(zs):
        turned[i] = [(rotate(typ, r, t, None, pos)[0].double().cpu(), bound(t)) for t in (x + z, x - z)]
    for i in range(dim // 2):
        r.freq[i] = -r.freq[i]
    grad, off = rotate(typ, r, y, None, pos)[0].double().cpu(), bound(y)
    y = y.double().cpu()
    for i, z in enumerate(zs):
        (a, ea), (b, eb) = turned[i]
        z = z.double().cpu()
        err = float(((a - b) * y).sum() - 2 * (z * grad).sum())
        assert abs(err) <= float(((ea + eb) * y.abs()).sum() + 2 * (z.abs() * off).sum()), (i, err)
        # and one pair alone, where errors cannot cancel: direction z in it, the loss its two values times y
        at = i % (dim // 2)
        pair = [2 * at, 2 * at + 1] if inter else [at, at + dim // 2]
        err = ((a - b) * y)[..., pair].sum(-1) - 2 * (z * grad)[..., pair].sum(-1)
        assert (err.abs() <= ((ea + eb) * y.abs())[..., pair].sum(-1) + 2 * (z.abs() * off)[..., pair].sum(-1)).all(), i


@ALL
def test_rotate_strides(typ):
    """Slices of a joint projection, heads before tokens, one row for all tokens; outputs in a joint tensor."""
    dt, n = TYPES[typ][0], 33
    joint = randn((n, 4 + 2 + 2, 48), dt, 4)
    pos, r = [5 * i for i in range(n)], rotary(40, 0)
    q, k = joint[:, :4], joint[:, 4:6]
    want_q, want_k = rotate(typ, r, q.contiguous(), k.contiguous(), pos)
    before = joint[:, 6:].clone()
    rotate(typ, r, q, k, pos, q, k)                   # in place inside the projection
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(joint[:, 6:], before)
    heads_first = randn((4, n, 48), dt, 5).transpose(0, 1)
    out = torch.empty(4, n, 48, dtype=dt, device=DEV).transpose(0, 1)
    rotate(typ, r, heads_first, None, pos, out)
    assert torch.equal(out, rotate(typ, r, heads_first.contiguous(), None, pos)[0])
    one = randn((1, 4, 48), dt, 6).expand(n, 4, 48)
    assert torch.equal(rotate(typ, r, one, None, pos)[0], rotate(typ, r, one.contiguous(), None, pos)[0])


# ---------------------------------------------------------------- into the cache

@ALL
@pytest.mark.parametrize("dim,page,rot,inter", [(32, 32, 32, 0), (64, 64, 20, 0), (64, 64, 64, 1), (96, 32, 50, 1),
                                                (128, 128, 128, 0), (128, 32, 96, 0)])
def test_append_rotary_is_rotate_and_append(typ, dim, page, rot, inter):
    """Pools, byte for byte, and queries; slots out of range and rows that the sequence has no place for among them."""
    print("\n[gpu-case] append_rotary", typ, dim, page, rot, inter, flush=True)
    dt, lens, new = TYPES[typ][0], [70, 31, 0, 1, 300, 33], [45, 31, 2, 1, 200, 40]
    n, heads = sum(new) + 3, 6
    a, b = (Cache(2, dim, page, 40, 8, 12) for _ in range(2))
    for c in (a, b):
        c.place(lens)
        c.pool.copy_(torch.randint(0, 120, c.pool.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(1)))
    joint = randn((n, heads + 4, dim), dt, 2)
    q, k, v = joint[:, :heads], joint[:, heads:heads + 2], joint[:, heads + 2:]
    r = rotary(rot, inter, 1.0, 10000.0, 4.0)
    seqs, cu = [0, 1, 2, 3, 4, 5, 12345, -1], offsets(new) + [sum(new) + 1, sum(new) + 3]
    o = offsets(new)
    pos, live = [], []
    for i, s in enumerate(new):
        pos += [lens[i] - s + j for j in range(s)]
    live = [p >= 0 for p in pos] + [False] * 3
    pos += [0] * 3
    want_q, want_k = rotate(typ, r, q, k, pos)
    ts, tc = i32(seqs), i32(cu)
    I.ios_cache_append(a.c, 0, TYPES[typ][1], toks(want_k), toks(v), 8, ts.data_ptr(), tc.data_ptr(), stream())
    qo = torch.full((n, heads, dim), 7.0, dtype=dt, device=DEV)
    I.ios_cache_append_rotary(b.c, 0, TYPES[typ][1], r, toks(q), toks(qo), heads, toks(k), toks(v), 8, ts.data_ptr(),
                              tc.data_ptr(), stream())
    torch.cuda.synchronize()
    assert torch.equal(a.pool, b.pool)
    rows = torch.tensor(live)
    assert torch.equal(qo[rows], want_q[rows]) and (qo[~rows] == 7).all()
    gk, gv = b.read([0], [45])
    assert equal(gk, held(want_k[:45])) and equal(gv, held(v[:45]))
    # without queries, and queries in place
    before = b.pool.clone()
    I.ios_cache_append_rotary(b.c, 0, TYPES[typ][1], r, None, None, 0, toks(k), toks(v), 8, ts.data_ptr(), tc.data_ptr(),
                              stream())
    I.ios_cache_append_rotary(b.c, 0, TYPES[typ][1], r, toks(q), toks(q), heads, toks(k), toks(v), 8, ts.data_ptr(),
                              tc.data_ptr(), stream())
    torch.cuda.synchronize()
    assert torch.equal(b.pool, before) and torch.equal(q[rows], want_q[rows])


def test_append_rotary_far_positions():
    """Single tokens behind a long sequence, more heads of queries than a workgroup takes."""
    c = Cache(1, 64, 256, 600, 2, 500)
    c.place([120001, 7])
    q, k, v = (randn((2, h, 64), torch.bfloat16, s) for s, h in ((1, 11), (2, 1), (3, 1)))
    r, qo, seqs, cu = rotary(64), torch.empty_like(q), i32([0, 1]), i32([0, 1, 2])
    I.ios_cache_append_rotary(c.c, 0, I.IOS_BF16, r, toks(q), toks(qo), 11, toks(k), toks(v), 2, seqs.data_ptr(),
                              cu.data_ptr(), stream())
    torch.cuda.synchronize()
    want_q, want_k = rotate("bf16", r, q, k, [120000, 6])
    assert torch.equal(qo, want_q)
    gk, gv = c.read([0, 1], [1, 1])
    assert equal(gk, held(want_k)) and equal(gv, held(v))


def test_append_rotary_missing_page_and_nan():
    c = Cache(1, 32, 32, 4, 1, 3)
    c.place([64])
    c.table[0, 1] = 999
    q, k, v = (randn((40, 1, 32), torch.float32, s) for s in (1, 2, 3))
    k[3, 0, 5] = math.nan                           # its whole group of 32 is NaN, as without positions
    r, qo, seqs, cu = rotary(32), torch.full_like(q, 7.0), i32([0]), i32([0, 40])
    before = c.pool.clone()
    I.ios_cache_append_rotary(c.c, 0, I.IOS_F32, r, toks(q), toks(qo), 1, toks(k), toks(v), 1, seqs.data_ptr(),
                              cu.data_ptr(), stream())
    torch.cuda.synchronize()
    want_q, want_k = rotate("f32", r, q, k, list(range(24, 64)))
    assert torch.equal(qo, want_q)                  # queries need no page
    gk, _ = c.read([0], [64])
    assert equal(gk[24:32], held(want_k[:8])) and torch.isnan(gk[27]).all()
    other = [p for p in range(4) if p != int(c.table[0, 0])]
    assert torch.equal(c.pool[:, other], before[:, other])


@ALL
@pytest.mark.parametrize("most", [1, 5, 33, 64])
def test_keep_is_append_of_the_rows(typ, most):
    print("\n[gpu-case] keep", typ, most, flush=True)
    dt, rng = TYPES[typ][0], np.random.default_rng(most)
    lens, n = [90, 31, 64, 5, 200, 33, 0], 50
    count = [0, min(most, 7), most, most + 9, min(most, 40), -3, 1]
    seqs = [0, 1, 2, 3, 4, -1, 12345]
    path = rng.integers(0, n, (7, most))
    a, b = (Cache(2, 64, 32, 40, 7, 12) for _ in range(2))
    for c in (a, b):
        c.place(lens)
        c.pool.copy_(torch.randint(0, 120, c.pool.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(1)))
    joint = randn((n, 4, 64), dt, 2)
    k, v = joint[:, :2], joint[:, 2:]
    kept = [min(max(x, 0), most) for x in count]
    rows = [int(x) for i in range(5) for x in path[i, :kept[i]]]
    if rows:
        a.append(k[rows], v[rows], seqs[:5], kept[:5], typ)
    tp, tc, ts = i32(path.tolist()), i32(count), i32(seqs)
    I.ios_cache_keep(b.c, 0, TYPES[typ][1], toks(k), toks(v), 7, ts.data_ptr(), tp.data_ptr(), most, tc.data_ptr(), stream())
    torch.cuda.synchronize()
    assert torch.equal(a.pool, b.pool)


def test_keep_rows_out_of_range():
    """A row that is not there makes its token 0, the others are as they should be."""
    c = Cache(1, 32, 32, 4, 1, 4)
    c.place([10])
    k, v = randn((6, 1, 32), torch.float16, 1), randn((6, 1, 32), torch.float16, 2)
    path, count, seqs = i32([[5, -1, 0, 6, 1 << 30, 2]]), i32([6]), i32([0])
    I.ios_cache_keep(c.c, 0, I.IOS_F16, toks(k), toks(v), 1, seqs.data_ptr(), path.data_ptr(), 6, count.data_ptr(), stream())
    torch.cuda.synchronize()
    gk, gv = c.read([0], [6])
    for j, row in enumerate([5, None, 0, None, None, 2]):
        if row is None:
            assert (gk[j] == 0).all() and (gv[j] == 0).all()
        else:
            assert equal(gk[j:j + 1], held(k[row:row + 1])) and equal(gv[j:j + 1], held(v[row:row + 1]))
    none = toks(k[:0])
    I.ios_cache_keep(c.c, 0, I.IOS_F16, none, none, 1, seqs.data_ptr(), path.data_ptr(), 6, count.data_ptr(), stream())
    torch.cuda.synchronize()
    assert (c.read([0], [6])[0] == 0).all()


# ---------------------------------------------------------------- attention of drafts

def forest(n, rng, kind):
    if kind == "chain":
        return [j - 1 for j in range(n)]
    if kind == "roots":
        return [-1] * n
    return [int(rng.integers(-1, j)) if j else -1 for j in range(n)]


def visible(parent):
    """[row][draft], a parent that is not an earlier draft's is none."""
    n = len(parent)
    m = torch.zeros(n, n, dtype=torch.bool)
    for j in range(n):
        a = j
        while True:
            m[j, a] = True
            if not 0 <= parent[a] < a:
                break
            a = parent[a]
    return m


def tree_reference(typ, q, kc, vc, kd, vd, see, scale):
    """Rows q [n][d] over the cached keys and values (z, s, c each) of one head and its drafts: result, log-sum-exp, and
    bounds of both.  Values that a row does not see take no part."""
    q, kd, vd = q.double().cpu(), kd.double().cpu(), vd.double().cpu()
    (kz, ks, kcode), (vz, vs, vcode) = kc, vc
    m, d = len(kz), q.shape[1]
    fin = torch.isfinite(vd)
    v0, k0 = torch.where(fin, vd, 0.0), kd.nan_to_num(0.0, 0.0, 0.0)
    s = scale * torch.cat([q @ (kz + ks * kcode).T, torch.where(see, q @ k0.T, -math.inf / scale if scale else -math.inf)], 1)
    s[:, m:] = torch.where(see, s[:, m:], -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None]).nan_to_num(0.0)
    pc, pd = p[:, :m], p[:, m:]
    out = pc @ (vz + vs * vcode) + pd @ v0
    bad = see.double()
    nan, up, dn = (bad @ x.double() > 0 for x in (torch.isnan(vd), vd == math.inf, vd == -math.inf))
    out = torch.where(up, math.inf, torch.where(dn, -math.inf, out))
    out = torch.where(nan | (up & dn), math.nan, out)
    far = (q.abs() @ (kz.abs() + 15 * ks).T) * (2.0 ** -22 + 2.0 ** -24 * (d + 8) + (2.0 ** -11 if typ == "bf16" else 0.0))
    near = torch.where(see, q.abs() @ k0.abs().T, 0.0) * 2.0 ** -24 * (d + 10)
    e = abs(scale) * torch.cat([far, near], 1).amax(1, keepdim=True) if m + len(kd) else torch.zeros(len(q), 1)
    ac, ad = pc @ (vz.abs() + 15 * vs), pd @ v0.abs()
    ps, a = pc @ vs, ac + ad
    top = float((vz + vs * vcode).abs().max()) if m else 0.0
    # a row's largest weight is 2^9 at least where 16 bits hold it, so one is off by half a step or by 2^-25 at most: 2^-34
    # of the largest for each key, and that is at most the sum of them
    w, summed = {"bf16": (2.0 ** -10 * ac + 2.0 ** -34 * m * top, a), "f16": (2.0 ** -20 * ac + 2.0 ** -34 * m * top, a),
                 "f32": (2.0 ** -24 * 15 * ps, a)}[typ]
    r = 33 * -(-m // 128) + 128 + 8 + 40 + 128
    fine = torch.where(torch.isfinite(out), out, 0.0).abs()
    bound = TYPES[typ][2] * fine + 2.0 ** -25 + (2 * e + 2.0 ** -17) * a + w + 2.0 ** -16 * ad + 2.0 ** -24 * r * (summed + fine)
    return out, lse, bound, e[:, 0] + 2.0 ** -17 + 2.0 ** -24 * r + 2.0 ** -22 * (1 + lse.abs())


def tree(typ, c, q, k, v, seqs, cu, parent, most, max_keys=0, work=True, scale=None, layer=0):
    d = desc(typ, q.shape[1], c.c.kv_heads, c.c.head_dim, len(seqs), 0, max_keys, scale)
    n = I.ios_attn_tree_work_bytes(d, q.shape[0], most) if work else 0
    w = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV)
    out = torch.empty(q.shape, dtype=q.dtype, device=DEV).fill_(7.0)
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device=DEV)
    ts, tc, tp = i32(seqs), i32(cu), i32(parent)
    I.ios_attn_tree(c.c, layer, d, toks(q), toks(k), toks(v), toks(out), lse.data_ptr(), ts.data_ptr(), tc.data_ptr(),
                    tp.data_ptr(), most, w.data_ptr() if n else 0, n, stream())
    torch.cuda.synchronize()
    return out, lse, d.scale


def check_tree(typ, c, q, k, v, seqs, drafts, parents, hk, hv, most=None, **kw):
    """hk, hv: z, s and c of every slot's keys and values [tokens][heads][dim]."""
    most = max(drafts + [1]) if most is None else most
    flat = [p for t in parents for p in t]
    flat += [-1] * (q.shape[0] - len(flat))
    out, lse, scale = tree(typ, c, q, k, v, seqs, offsets(drafts), flat, most, **kw)
    o, ratio = offsets(drafts), q.shape[1] // c.c.kv_heads
    empty = [torch.zeros(0, c.c.kv_heads, c.c.head_dim, dtype=torch.float64)] * 3
    for i, s in enumerate(seqs):
        n = min(drafts[i], most)
        rows, see = slice(o[i], o[i] + n), visible(parents[i][:n])
        kk, vv = (hk[s], hv[s]) if 0 <= s < len(hk) else (empty, empty)
        for h in range(q.shape[1]):
            g = h // ratio
            ref, l64, bound, far = tree_reference(typ, q[rows, h], [x[:, g] for x in kk], [x[:, g] for x in vv], k[rows, g],
                                                  v[rows, g], see, scale)
            got, gl = out[rows, h].double().cpu(), lse[h, rows].double().cpu()
            same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))
            err = (got - ref).abs()
            assert (same | (err <= bound)).all(), (i, h, float((err / bound)[~same].max()))
            assert ((gl - l64).abs() <= far).all(), (i, h, gl, l64)
        assert (out[o[i] + n:o[i + 1]] == 7).all() and (lse[:, o[i] + n:o[i + 1]] == 7).all()
    assert (out[o[-1]:] == 7).all()                  # rows of no sequence
    return out


def cached(kv, dim, page, lens, seed, scale=1.0):
    """A cache with these sequences; the values' mean drifts along each, so that no part of it can be missed."""
    c = Cache(kv, dim, page, sum(-(-m // page) for m in lens) + 3, len(lens) + 1, max(-(-m // page) for m in lens) + 1)
    c.place(lens, seed)
    k, v = (randn((sum(lens), kv, dim), torch.float32, s) for s in (seed, seed + 1))
    v += torch.cat([torch.linspace(-1.0, 1.0, m) for m in lens])[:, None, None].to(DEV) * scale
    if sum(lens):
        c.append(k, v, list(range(len(lens))), lens, "f32")
    o = offsets(lens)
    hk, hv = ([[t[o[i]:o[i + 1]] for t in quantised(x)] for i in range(len(lens))] for x in (k, v))
    return c, hk, hv


@ALL
@pytest.mark.parametrize("dim,page,kv,ratio,kind", [(32, 32, 2, 1, "tree"), (64, 64, 1, 8, "chain"), (96, 32, 2, 5, "tree"),
                                                    (128, 128, 2, 4, "tree"), (128, 32, 1, 16, "roots"), (64, 256, 1, 3, "chain"),
                                                    (32, 64, 1, 20, "tree")])
def test_tree(typ, dim, page, kv, ratio, kind):
    """Every length around a tile, empty sequences and slots out of range, one draft to 64, a sequence without any."""
    print("\n[gpu-case] tree", typ, dim, page, kv, ratio, kind, flush=True)
    lens = [0, 1, 31, 32, 33, 64, 300, 1100]
    c, hk, hv = cached(kv, dim, page, lens, 3)
    seqs, drafts = [7, 0, 1, 2, -1, 3, 4, 5, 6, 12345], [17, 33, 1, 2, 64, 0, 31, 16, 48, 5]
    rng = np.random.default_rng(dim + ratio)
    parents = [forest(n, rng, kind) for n in drafts]
    n = sum(drafts) + 3
    dt = TYPES[typ][0]
    q, k, v = randn((n, kv * ratio, dim), dt, 5), randn((n, kv, dim), dt, 6), randn((n, kv, dim), dt, 7, 3.0)
    q[2] *= 20.0                                     # one key far ahead of the others
    q[3] *= 2.0 ** -12
    q[60, 0] = 0.0
    k[n - 3:], v[n - 3:] = math.nan, math.nan        # rows of no sequence
    for kw in (dict(), dict(work=False), dict(max_keys=1100)):
        check_tree(typ, c, q, k, v, seqs, drafts, parents, hk, hv, **kw)


@ALL
@pytest.mark.parametrize("dim,kv,ratio,drafts", [(128, 2, 8, 32), (64, 1, 4, 64), (96, 1, 1, 7), (128, 1, 1, 1), (32, 2, 3, 21)])
def test_tree_long(typ, dim, kv, ratio, drafts):
    """Caches that are spread over workgroups, of unequal lengths, with a bound that is right, wrong or unknown."""
    print("\n[gpu-case] tree long", typ, dim, kv, ratio, drafts, flush=True)
    lens = [9000, 2049, 40]
    c, hk, hv = cached(kv, dim, 64, lens, 9)
    rng = np.random.default_rng(1)
    counts = [drafts, max(1, drafts // 2), drafts]
    parents, n, dt = [forest(m, rng, "tree") for m in counts], sum(counts), TYPES[typ][0]
    q, k, v = randn((n, kv * ratio, dim), dt, 5), randn((n, kv, dim), dt, 6), randn((n, kv, dim), dt, 7)
    check_tree(typ, c, q, k, v, [0, 1, 2], counts, parents, hk, hv, max_keys=9000)
    check_tree(typ, c, q, k, v, [1, 2, 0], counts, parents, hk, hv, max_keys=100)
    check_tree(typ, c, q, k, v, [0, 1, 2], counts, parents, hk, hv, scale=-0.2)


@ALL
def test_tree_strides_and_odd_parents(typ):
    """Slices of a joint projection, heads first, one key for all; parents that are themselves, later, out of range."""
    dt = TYPES[typ][0]
    c, hk, hv = cached(2, 64, 32, [50, 20], 11)
    drafts = [9, 12]
    parents = [[0, 5, 1, -7, 3, 4, 99, 2, 1 << 30], [-1, 0, 1, 1, 4, 11, 5, 6, 20, 8, 9, 10]]
    joint = randn((21, 4 + 2 + 2, 64), dt, 4)
    q, k, v = joint[:, :4], joint[:, 4:6], joint[:, 6:]
    check_tree(typ, c, q, k, v, [0, 1], drafts, parents, hk, hv)
    check_tree(typ, c, randn((4, 21, 64), dt, 5).transpose(0, 1), randn((2, 21, 64), dt, 6).transpose(0, 1), v, [1, 0], drafts,
               parents, hk, hv)
    check_tree(typ, c, q, k[:1].expand(21, 2, 64), v[:, :1].expand(21, 2, 64), [0, 1], drafts, parents, hk, hv)
    # fewer drafts than the sequences have: the rows past them are left alone
    check_tree(typ, c, q, k, v, [0, 1], drafts, parents, hk, hv, most=7)


@ALL
def test_tree_hidden_infinities_and_nan(typ):
    """Drafts that a row does not see never change it; infinities and NaN that it sees are in its result."""
    dt = TYPES[typ][0]
    c, hk, hv = cached(1, 64, 32, [1300, 0], 13)
    drafts, parents = [40, 40], [forest(40, np.random.default_rng(2), "tree")] * 2
    q, k, v = randn((80, 3, 64), dt, 5), randn((80, 1, 64), dt, 6), randn((80, 1, 64), dt, 7)
    clean, lse0, _ = tree(typ, c, q, k, v, [0, 1], [0, 40, 80], parents[0] * 2, 40, max_keys=1300)
    for work in (True, False):
        v2 = v.clone()
        v2[5, 0, 3], v2[33, 0, 5], v2[44, 0, 6], v2[73, 0, 7], v2[73, 0, 6] = math.nan, math.inf, -math.inf, math.inf, math.inf
        check_tree(typ, c, q, k, v2, [0, 1], drafts, parents, hk, hv, max_keys=1300, work=work)
        # an infinity stays one however little its key weighs
        k2, q2 = k.clone(), q.clone()
        q2[:, :, 0], k2[:, 0, 0], k2[33, 0, 0] = 40.0, 3.0, -30.0
        got, _, _ = tree(typ, c, q2, k2, v2, [0, 1], [0, 40, 80], parents[0] * 2, 40, max_keys=1300, work=work)
        see = visible(parents[0])[:, 33].to(DEV)
        assert (got[:40][see][:, :, 5] == math.inf).all() and torch.isfinite(got[:40][~see][:, :, 5]).all()
        # keys: rows that see a NaN are NaN, the others are as before to the bit
        k3, v3 = k.clone(), v.clone()
        k3[7] = math.nan
        got, lse, _ = tree(typ, c, q, k3, v, [0, 1], [0, 40, 80], parents[0] * 2, 40, max_keys=1300, work=work)
        see = torch.cat([visible(parents[0])[:, 7], torch.zeros(40, dtype=torch.bool)]).to(DEV)
        ref, lref, _ = tree(typ, c, q, k, v, [0, 1], [0, 40, 80], parents[0] * 2, 40, max_keys=1300, work=work)
        assert torch.isnan(got[see]).all() and torch.equal(got[~see], ref[~see]) and torch.equal(lse[:, ~see], lref[:, ~see])
        # the type's ends, hidden
        big = torch.finfo(dt).max
        k3[7], v3[7] = -big, big
        got, _, _ = tree(typ, c, q, k3, v3, [0, 1], [0, 40, 80], parents[0] * 2, 40, max_keys=1300, work=work)
        assert torch.equal(got[~see], ref[~see])
    assert torch.isfinite(clean).all()


@ALL
def test_tree_largest_values_stay_finite(typ):
    """Values at the type's ends give means within it, alone and beside cached ones."""
    dt = TYPES[typ][0]
    big = torch.finfo(dt).max
    c, hk, hv = cached(1, 32, 32, [1100, 0], 15)
    q, k = randn((64, 2, 32), dt, 5), randn((64, 1, 32), dt, 6)
    v = torch.full((64, 1, 32), big, dtype=dt, device=DEV)
    v[:, :, 1::2] = -big
    chain = [j - 1 for j in range(64)]
    for work in (True, False):
        out, _, _ = tree(typ, c, q, k, v, [1], [0, 64], chain, 64, max_keys=1100, work=work)
        ref = torch.full((64, 2, 32), float(big), dtype=torch.float64)
        ref[:, :, 1::2] *= -1
        got = out.double().cpu()
        assert torch.isfinite(got).all() and ((got - ref).abs() <= (TYPES[typ][2] + 2.0 ** -15) * big).all()
        out, _, _ = tree(typ, c, q, k, v, [0], [0, 64], chain, 64, max_keys=1100, work=work)
        for h in range(2):
            ref, _, bound, _ = tree_reference(typ, q[:, h], [x[:, 0] for x in hk[0]], [x[:, 0] for x in hv[0]], k[:, 0], v[:, 0],
                                              visible(chain), 1 / math.sqrt(32))
            err = (out[:, h].double().cpu() - ref).abs()
            assert torch.isfinite(out[:, h]).all() and (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("size,low", [(8.0, -110.0), (1.0, -200.0)])
def test_tree_large_value_of_no_weight(typ, size, low):
    """A value of 2^100 whose weight is e^-110 or less leaves the other keys' weights as exact as they were; one of 2^120 with
    a score of -20 is what its row comes to: cached scores, size times a normal number and a small one, stay below 45, so its
    weight is e^-65 / 2500 = 2^-106 at least."""
    dt = TYPES[typ][0]
    c, hk, hv = cached(1, 64, 64, [2500], 23)
    u = torch.zeros(64, device=DEV)
    u[5] = size
    q = (randn((6, 4, 64), torch.float32, 1, 0.125) + u).to(dt)
    k, v = randn((6, 1, 64), dt, 2, 0.25), randn((6, 1, 64), dt, 3)
    k[1, 0], v[1, 0, 7] = (low / size * u / size).to(dt), 2.0 ** 100
    k[4, 0], v[4, 0, 9] = (-20.0 / size * u / size).to(dt), -2.0 ** 120
    parents = [[-1, 0, 1, 1, 0, 4]]
    out = check_tree(typ, c, q, k, v, [0], [6], parents, hk, hv, max_keys=2500, scale=1.0)
    assert (out[1:4].abs() < 100).all() and (out[4:, :, 9] < -2.0 ** 13).all()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("large", [2.0 ** 104, 3.0e38, math.inf])
@pytest.mark.parametrize("lead", [4.0, -20.0])
@pytest.mark.parametrize("dim,kv,ratio,drafts,bound", [(64, 1, 4, 6, 2500), (32, 2, 1, 40, 2500), (96, 1, 16, 5, 2500),
                                                       (64, 8, 8, 8, 0)])
def test_tree_one_large_value_among_ordinary_ones(typ, large, lead, dim, kv, ratio, drafts, bound):
    """A draft with one very large value: the other values of the rows that see it, which are mostly the cache's, stay within
    the bounds of ordinary ones; rows that do not see it stay as they are to the bit.  Drafts score 4 (base 2) above the
    cached tokens, or 20 below; the cached values are 2 in the mean, and each of a workgroup's waves has an eighth of that."""
    print("\n[gpu-case] tree one large value", typ, large, lead, dim, kv, ratio, drafts, flush=True)
    dt, lens, who = TYPES[typ][0], [2500, 300], drafts - 2
    c = Cache(kv, dim, 64, 50, 3, 40)
    c.place(lens, 31)
    kc, vc = randn((2800, kv, dim), torch.float32, 31), randn((2800, kv, dim), torch.float32, 32) + 2.0
    c.append(kc, vc, [0, 1], lens, "f32")
    hk, hv = ([[t[:2500] for t in quantised(x)], [t[2500:] for t in quantised(x)]] for x in (kc, vc))
    parents = [forest(drafts, np.random.default_rng(drafts + i), "tree") for i in range(2)]
    parents[0][drafts - 1] = who
    flat, n, cu = parents[0] + parents[1], 2 * drafts, [0, drafts, 2 * drafts]
    q, k, v = randn((n, kv * ratio, dim), dt, 5, 0.25), randn((n, kv, dim), dt, 6), randn((n, kv, dim), dt, 7)
    q[:, :, 0], k[:, :, 0] = 4.0, lead * math.log(2.0) / (4.0 * 2.0 ** -5)
    big = v.clone()
    big[who, :, 9], big[drafts, 0, 3] = large, -large
    see = torch.zeros(n, dtype=torch.bool)
    see[:drafts], see[drafts:] = visible(parents[0])[:, who], visible(parents[1])[:, 0]
    assert see.any() and not see.all()
    for work in (True, False):
        clean, _, _ = tree(typ, c, q, k, v, [0, 1], cu, flat, drafts, max_keys=bound, work=work, scale=2.0 ** -5)
        got = check_tree(typ, c, q, k, big, [0, 1], [drafts] * 2, parents, hk, hv, max_keys=bound, work=work, scale=2.0 ** -5)
        assert torch.equal(got[~see.to(DEV)], clean[~see.to(DEV)])
        assert torch.isfinite(got[:, :, 10:]).all()


@pytest.mark.parametrize("typ", ["bf16", "f16"])
@pytest.mark.parametrize("bound", [5000, 0])
def test_tree_ragged_batch(typ, bound):
    """Shares that begin and end inside blocks of rows and sequences, with trees of every size: 64 rows a block where the
    lengths may be long, 32 where they may not."""
    rng = np.random.default_rng(3)
    lens = [int(x) for x in np.exp(rng.uniform(0, math.log(5000), 18))] + [0, 5000]
    drafts = [int(x) for x in rng.integers(0, 33, 20)]
    c, hk, hv = cached(2, 64, 32, lens, 29)
    parents, n = [forest(m, rng, "tree") for m in drafts], sum(drafts)
    dt = TYPES[typ][0]
    q, k, v = randn((n, 6, 64), dt, 5), randn((n, 2, 64), dt, 6), randn((n, 2, 64), dt, 7)
    order = [int(x) for x in rng.permutation(20)]
    check_tree(typ, c, q, k, v, order, drafts, parents, hk, hv, max_keys=bound)


def test_tree_more_sequences_than_threads():
    """1300 sequences, three for a thread that lays out the shares, some listed twice, some without drafts or tokens."""
    lens = [(37 * i) % 120 for i in range(40)]
    c, hk, hv = cached(1, 32, 32, lens, 31)
    drafts = [(i * i) % 4 for i in range(1300)]
    parents, n = [[j - 1 for j in range(m)] for m in drafts], sum(drafts)
    q, k, v = randn((n, 1, 32), torch.float16, 1), randn((n, 1, 32), torch.float16, 2), randn((n, 1, 32), torch.float16, 3)
    check_tree("f16", c, q, k, v, [(7 * i) % 43 - 1 for i in range(1300)], drafts, parents, hk, hv)


@pytest.mark.parametrize("work", [True, False])
@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, 1e-35, -1e-35])
def test_tree_large_scores_of_a_small_scale(typ, scale, work):
    """Scores of 10^35 and more weigh as the definition says, also times 0."""
    dt = TYPES[typ][0]
    c, hk, hv = cached(1, 32, 32, [1100, 40], 43)
    parents = [forest(9, np.random.default_rng(i), "tree") for i in range(2)]
    q, k, v = (randn((18, h, 32), torch.float32, s, size).to(dt) for h, s, size in ((3, 1, 1e17), (1, 2, 1e17), (1, 3, 1.0)))
    check_tree(typ, c, q, k, v, [0, 1], [9, 9], parents, hk, hv, max_keys=1100, work=work, scale=scale)


@pytest.mark.parametrize("work", [True, False])
@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("where", ["cache", "drafts"])
def test_tree_scores_beyond_float32_are_not_zeros(typ, where, work):
    """Where scores times log2(e) leave float32's range there is no result; it reads as NaN, not as a row of zeros."""
    dt = TYPES[typ][0]
    c = Cache(1, 32, 32, 40, 1, 36)
    c.place([1100])
    k = torch.full((1100, 1, 32), 2.0, device=DEV)
    k[1::2] = 1.0
    c.append(k, randn((1100, 1, 32), torch.float32, 2), [0], [1100], "f32")
    q = torch.full((6, 2, 32), 2.0 ** 122 if where == "cache" else 2.5e18, dtype=dt, device=DEV)      # scores of 3e38
    kd = torch.full((6, 1, 32), 0.0 if where == "cache" else 2.5e18, dtype=dt, device=DEV)
    out, lse, _ = tree(typ, c, q, kd, randn((6, 1, 32), dt, 3), [0], [0, 6], [-1, 0, 1, 1, 3, -1], 6, max_keys=1100, work=work,
                       scale=1.5)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("work", [True, False])
def test_tree_more_rows_than_a_workgroup_each(work):
    """8192 sequences under 32 drafts of 32 heads, 2^23 rows in all; every four sequences are the same."""
    n, drafts, heads, dim, lens = 8192, 32, 32, 32, [1100, 40, 0, 300]
    print("\n[gpu-case] tree of 2^23 rows", work, flush=True)
    c, hk, hv = cached(1, dim, 32, lens, 41)
    parents = [forest(drafts, np.random.default_rng(i), kind) for i, kind in enumerate(["tree", "chain", "roots", "tree"])]
    q, k, v = (randn((4 * drafts, h, dim), torch.float16, s) for h, s in ((heads, 1), (1, 2), (1, 3)))
    out, lse, scale = tree("f16", c, *(t.repeat(n // 4, 1, 1) for t in (q, k, v)), [0, 1, 2, 3] * (n // 4),
                           [drafts * i for i in range(n + 1)], [p for t in parents for p in t] * (n // 4), drafts, max_keys=1100,
                           work=work)
    out, lse = out.view(n // 4, 4, drafts, heads, dim), lse.view(heads, n // 4, 4, drafts)
    for i in range(4):
        rows, see = slice(drafts * i, drafts * i + drafts), visible(parents[i])
        for h in range(heads):
            ref, l64, bound, far = (t.to(DEV) for t in tree_reference("f16", q[rows, h], [x[:, 0] for x in hk[i]],
                                                                      [x[:, 0] for x in hv[i]], k[rows, 0], v[rows, 0], see, scale))
            err = (out[:, i, :, h].double() - ref).abs()
            assert (err <= bound).all(), (i, h, float((err / bound).max()))
            assert ((lse[h, :, i].double() - l64).abs() <= far).all(), (i, h)


@ALL
@pytest.mark.parametrize("lead", [11.5, 18.0])
def test_tree_long_tail(typ, lead):
    """One key far ahead of many equal ones, in the cache and among the drafts."""
    n = 50000 if lead > 12 else 6000
    for where in ("cache", "draft"):
        c = Cache(1, 32, 256, 200, 1, 200)
        c.place([n])
        k, v = torch.zeros(n, 1, 32, device=DEV), torch.ones(n, 1, 32, device=DEV)
        dt = TYPES[typ][0]
        kd, vd = torch.zeros(3, 1, 32, dtype=dt, device=DEV), torch.ones(3, 1, 32, dtype=dt, device=DEV)
        if where == "cache":
            k[77, 0, 0], v[77] = lead, -1.0
        else:
            kd[0, 0, 0], vd[0] = lead, -1.0
        c.append(k, v, [0], [n], "f32")
        q = torch.zeros(3, 2, 32, dtype=dt, device=DEV)
        q[:, :, 0] = 1.0
        check_tree(typ, c, q, kd, vd, [0], [3], [[-1, 0, 1]], [[x for x in quantised(k)]], [[x for x in quantised(v)]],
                   max_keys=n, scale=1.0)


@ALL
def test_tree_one_draft_is_single_token_attention(typ):
    """A draft whose key and value are exact in the cache: attention over the cache that holds it agrees."""
    from test_gpu_decoder import decode
    dt = TYPES[typ][0]
    c, hk, hv = cached(2, 64, 32, [700], 17)
    k1 = (torch.arange(64, device=DEV) % 16).to(dt).expand(1, 2, 64)        # 0 .. 15 a group: scale 1, zero 0
    v1 = (15 - torch.arange(64, device=DEV) % 16).to(dt).expand(1, 2, 64)
    q = randn((1, 6, 64), dt, 5)
    a, la, _ = tree(typ, c, q, k1, v1, [0], [0, 1], [-1], 1)
    c.reserve([0], [1])
    c.append(k1.contiguous(), v1.contiguous(), [0], [1], typ)
    b, lb, _ = decode(c, typ, q, [0])
    assert torch.allclose(la, lb, atol=2.0 ** -9 if typ == "bf16" else 2.0 ** -16)
    size = 16.0
    assert ((a.double() - b.double()).abs() <= {"bf16": 2.0 ** -7, "f16": 2.0 ** -10, "f32": 2.0 ** -16}[typ] * size).all()


def test_tree_bad_offsets_and_many_sequences():
    """Offsets that leave the tensors or descend are clipped; the first sequence may begin later."""
    c, hk, hv = cached(1, 32, 32, [5 * (i % 9) for i in range(150)], 19)
    dt, drafts = torch.float16, [(3 * i) % 5 for i in range(150)]
    n = sum(drafts)
    q, k, v = randn((n + 20, 2, 32), dt, 1), randn((n + 20, 1, 32), dt, 2), randn((n + 20, 1, 32), dt, 3)
    parents = [[j - 1 for j in range(m)] for m in drafts]
    check_tree("f16", c, q, k, v, list(range(150)), drafts, parents, hk, hv)
    flat = [-1] * (n + 20)
    out, _, _ = tree("f16", c, q, k, v, [1, 2, 3], [13, 16, 1000000, -5], flat, 64)
    assert (out[:13] == 7).all() and (out[13:16] != 7).any() and (out[80 + 13:] == 7).all()
    out, _, _ = tree("f16", c, q, k, v, [1, 2], [50, 20, 10], flat, 64)
    assert (out == 7).all()


def test_tree_in_a_graph_with_other_lengths():
    """One recorded call, replayed with other cached lengths, trees and lists: the shares are laid out anew each time."""
    lens = [4000, 1, 900, 2600]
    c, hk, hv = cached(2, 64, 32, lens, 37)
    rng = np.random.default_rng(5)
    n, most, dt = 96, 32, torch.float16
    q, k, v = randn((n, 8, 64), dt, 5), randn((n, 2, 64), dt, 6), randn((n, 2, 64), dt, 7)
    d = desc("f16", 8, 2, 64, 3, 0, 4000)
    size = I.ios_attn_tree_work_bytes(d, n, most)
    work = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    seqs, cu, parent = i32([0, 1, 2]), i32([0, 0, 0, 0]), i32([-1] * n)

    def call(o, w):
        I.ios_attn_tree(c.c, 0, d, toks(q), toks(k), toks(v), toks(o), 0, seqs.data_ptr(), cu.data_ptr(), parent.data_ptr(),
                        most, w.data_ptr(), size, stream())
    call(out, work[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out, work[0])
    for i in range(8):
        drafts = [int(x) for x in rng.integers(0, 33, 3)]
        order = [int(x) for x in rng.permutation(4)[:3]]
        parents = [forest(m, rng, "tree") for m in drafts]
        flat = [p for t in parents for p in t]
        seqs.copy_(i32(order)), cu.copy_(i32(offsets(drafts))), parent.copy_(i32(flat + [-1] * (n - len(flat))))
        out.fill_(7.0), again.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        call(again, work[1])
        torch.cuda.synchronize()
        assert torch.equal(out, again) and (out[sum(drafts):] == 7).all(), i
        check_tree("f16", c, q, k, v, order, drafts, parents, hk, hv, max_keys=4000)


# ---------------------------------------------------------------- offsets that pass 32 bits

def test_pool_beyond_32_bits():
    """Drafts over, rotated appends into and drafts kept in pages that lie more than 4 GiB apart."""
    c = Cache(8, 128, 256, 16000, 2, 16)
    assert c.pool.numel() > 1 << 32
    lens = [3000, 500]
    c.place(lens, 3)
    assert int(c.table[c.table >= 0].max()) * c.pool.shape[2] > 1 << 32
    x, v = (randn((3500, 8, 128), torch.bfloat16, s) for s in (1, 2))
    r, seqs, cu = rotary(128), i32([0, 1]), i32([0, 3000, 3500])
    q = randn((3500, 8, 128), torch.bfloat16, 4)
    qo = torch.empty_like(q)
    I.ios_cache_append_rotary(c.c, 0, I.IOS_BF16, r, toks(q), toks(qo), 8, toks(x), toks(v), 2, seqs.data_ptr(), cu.data_ptr(),
                              stream())
    torch.cuda.synchronize()
    want_q, k = rotate("bf16", r, q, x, list(range(3000)) + list(range(500)))
    gk, gv = c.read([0, 1], lens)
    assert torch.equal(qo, want_q) and equal(gk, held(k)) and equal(gv, held(v))
    hk, hv = ([[t[:3000] for t in quantised(y.float())], [t[3000:] for t in quantised(y.float())]] for y in (k, v))
    parents = [forest(6, np.random.default_rng(i), "tree") for i in range(2)]
    qd, kd, vd = (randn((12, 8, 128), torch.bfloat16, s) for s in (5, 6, 7))
    for work in (True, False):
        check_tree("bf16", c, qd, kd, vd, [0, 1], [6, 6], parents, hk, hv, max_keys=3000, work=work)
    path, count = i32([[0, 2, 5], [6, 7, -1]]), i32([3, 2])
    I.ios_cache_keep(c.c, 0, I.IOS_BF16, toks(kd), toks(vd), 2, seqs.data_ptr(), path.data_ptr(), 3, count.data_ptr(), stream())
    torch.cuda.synchronize()
    gk, gv = c.read([0, 1], [3, 2])
    assert equal(gk, held(kd[[0, 2, 5, 6, 7]])) and equal(gv, held(vd[[0, 2, 5, 6, 7]]))


def test_rows_beyond_32_bits():
    """Rows 8 MiB apart, heads in turn 4 GiB apart: the same bits as from rows beside each other."""
    n, heads, kv, dim, dt = 600, 4, 2, 64, torch.bfloat16
    q, k, v = randn((n, heads, dim), dt, 1), randn((n, kv, dim), dt, 2), randn((n, kv, dim), dt, 3)
    room = torch.empty(n * (1 << 22), dtype=dt, device=DEV)

    def far(t, at):
        y = room.as_strided(t.shape, (1 << 22, t.shape[2], 1), at)
        y.copy_(t)
        return y
    fq, fk, fv, fo = far(q, 0), far(k, 4096), far(v, 8192), far(q, 12288)
    r, pos = rotary(dim), [3 * i for i in range(n)]
    want_q, want_k = rotate("bf16", r, q, k, pos)
    rotate("bf16", r, fq, fk, pos, fq, fk)
    assert torch.equal(fq, want_q) and torch.equal(fk, want_k)
    c, hk, hv = cached(kv, dim, 32, [1200, 70], 5)
    drafts, d = [15] * 40, desc("bf16", heads, kv, dim, 40, 0, 1200)
    seqs, cu, parent = i32([0, 1] * 20), i32(offsets(drafts)), i32([j - 1 for j in range(15)] * 40)
    size = I.ios_attn_tree_work_bytes(d, n, 15)
    work, out = torch.zeros(size, dtype=torch.uint8, device=DEV), torch.empty_like(q)
    for a, b, e, o in ((want_q, want_k, v, out), (fq, fk, fv, fo)):
        I.ios_attn_tree(c.c, 0, d, toks(a), toks(b), toks(e), toks(o), 0, seqs.data_ptr(), cu.data_ptr(), parent.data_ptr(), 15,
                        work.data_ptr(), size, stream())
    torch.cuda.synchronize()
    assert torch.equal(out, fo)
    del fq, fk, fv, fo, room
    # one head 4 GiB behind the other
    room = torch.empty(2, 1 << 31, dtype=dt, device=DEV)
    k2 = room.as_strided((n, kv, dim), (dim, 1 << 31, 1))
    k2.copy_(k)
    assert torch.equal(rotate("bf16", r, k2, None, pos, k2)[0], want_k)


# ---------------------------------------------------------------- the check of drafts

def walk(p, q, tokens, parent, accept, sample):
    """One sequence by the definition, in numpy's 64 bits: path, next token."""
    clean = lambda t: np.where(np.isfinite(t) & (t > 0), t, 0.0).astype(np.float64)  # noqa: E731
    p, n, vocab = clean(p), len(tokens), p.shape[1]
    q = clean(q) if q is not None else None
    if n == 0:
        return [], -1
    node, path = 0, [0]
    while True:
        rest, s, c, found = p[node].copy(), 1.0, 0.0, None
        for j in range(node + 1, n):
            x = tokens[j]
            if parent[j] != node or not 0 <= x < vocab:
                continue
            share = q[node, x] if q is not None else 1.0
            if float(accept[j]) * s * share < rest[x]:
                found = j
                break
            if q is not None:
                if s > 0:
                    c += s
                    rest = np.maximum(p[node] - c * q[node], 0.0)
                    s = rest.sum()
            else:
                s -= rest[x]
                rest[x] = 0.0
        if found is None:
            break
        node = found
        path.append(node)
    if rest.sum() == 0:
        rest = p[node]
    if rest.sum() == 0:
        return path, -1
    run = np.cumsum(rest)
    hit = np.nonzero((run > max(float(sample), 0.0) * run[-1]) & (rest > 0))[0]
    return path, int(hit[0]) if len(hit) else int(np.nonzero(rest)[0][-1])


def verify(typ, p, q, tokens, parent, cu, accept, sample, most):
    d = I.ios_verify_desc(TYPES[typ][1], len(cu) - 1, p.shape[1], most)
    size = I.ios_verify_work_bytes(d)
    work = torch.full((max(size, 16),), 255, dtype=torch.uint8, device=DEV)
    n = len(cu) - 1
    path, count, following = i32([[77] * most] * n), i32([77] * n), i32([77] * n)
    a, b, c = i32(tokens), i32(parent), i32(cu)
    rows = lambda t: I.ios_rows(t.data_ptr(), t.shape[0], t.stride(0))  # noqa: E731
    I.ios_verify(d, rows(p), rows(q) if q is not None else None, a.data_ptr(), b.data_ptr(), c.data_ptr(), accept.data_ptr(),
                 sample.data_ptr(), path.data_ptr(), count.data_ptr(), following.data_ptr(), work.data_ptr(), size, stream())
    torch.cuda.synchronize()
    return path, count, following


def check_verify(typ, p, q, tokens, parents, drafts, accept, sample, most=None):
    most = max(drafts + [1]) if most is None else most
    flat = [x for t in parents for x in t]
    path, count, following = verify(typ, p, q, tokens, flat, offsets(drafts), accept, sample, most)
    o, pn = offsets(drafts), p.float().cpu().numpy()
    qn = q.float().cpu().numpy() if q is not None else None
    for i, m in enumerate(drafts):
        rows = slice(o[i], o[i] + min(m, most))
        want, nxt = walk(pn[rows], qn[rows] if q is not None else None, tokens[rows], flat[rows], accept[rows].tolist(),
                         float(sample[i]))
        want = [o[i] + j for j in want]
        assert count[i].item() == len(want) and path[i].tolist() == want + [-1] * (most - len(want)), i
        assert following[i].item() == nxt, i
    return count


def spread(rows, vocab, typ, seed, far=1.0):
    g = torch.Generator().manual_seed(seed)
    x = 3.0 * torch.randn(rows, vocab, generator=g)
    p = torch.softmax(x, 1)
    q = torch.softmax(x + far * torch.randn(rows, vocab, generator=g), 1)
    return p.to(TYPES[typ][0]).to(DEV), q.to(TYPES[typ][0]).to(DEV)


def drawn(q, parents, drafts, seed):
    """Tokens from the parents' rows of q."""
    o, before = offsets(drafts), []
    for i, t in enumerate(parents):
        before += [o[i] + (j if 0 <= j < len(t) else 0) for j in t]
    if not before:
        return []
    return torch.multinomial(q.float().cpu()[before], 1, generator=torch.Generator().manual_seed(seed)).flatten().tolist()


def uniform(n, seed):
    return torch.rand(n, generator=torch.Generator().manual_seed(seed)).to(DEV)


@ALL
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("vocab", [1, 2, 7, 64, 513, 8191, 8192, 8193, 40009])
def test_verify(typ, given, vocab):
    """Chains, trees and bare rows, one to 64 a sequence, and sequences without any."""
    print("\n[gpu-case] verify", typ, given, vocab, flush=True)
    rng = np.random.default_rng(vocab)
    drafts = [1, 5, 0, 64, 9, 2, 33, 0] if vocab < 8000 else [1, 6, 0, 17, 3]
    parents = [forest(m, rng, "chain" if i % 2 else "tree") for i, m in enumerate(drafts)]
    parents = [[-1] + [max(x, 0) for x in t[1:]] if t else [] for t in parents]        # behind row 0, all of them
    p, q = spread(sum(drafts), vocab, typ, vocab)
    tokens = drawn(q, parents, drafts, 3)
    counts = []
    for seed in range(4):
        counts += check_verify(typ, p, q if given else None, tokens, parents, drafts, uniform(sum(drafts), seed),
                               uniform(len(drafts), 50 + seed)).tolist()
    if vocab > 2 and (given or vocab < 8000):              # a certain draft stands as often as p says: hardly ever here
        assert max(counts) > 1 and min(c for c in counts if c) == 1                    # some stand, some do not


@ALL
@pytest.mark.parametrize("given", [True, False])
def test_verify_large_vocabulary_and_strides(typ, given):
    """Rows of an odd length that start at any element, a stride between them, and one row for every draft."""
    vocab, drafts = 200003, [6, 9]
    parents = [[-1, 0, 0, 0, 1, 1], [j - 1 for j in range(9)]]
    p, q = spread(15, vocab + 5, typ, 1, 2.0)
    p, q = p[:, 3:3 + vocab], q[:, 2:2 + vocab]
    tokens = drawn(q, parents, drafts, 3)
    for seed in range(3):
        check_verify(typ, p, q if given else None, tokens, parents, drafts, uniform(15, seed), uniform(2, 9 + seed))
    check_verify(typ, p[4:5].expand(15, vocab), q[:1].expand(15, vocab) if given else None, tokens, parents, drafts,
                 uniform(15, 7), uniform(2, 8))


@pytest.mark.parametrize("given", [False, True])
def test_verify_largest_vocabulary(given):
    """2^31 - 1 tokens, all but four without a probability: the draw is from what a rejected draft leaves, not from p."""
    vocab = 2 ** 31 - 1
    p = torch.zeros(1, vocab, dtype=torch.bfloat16, device=DEV)
    p[0, 5], p[0, 77], p[0, 2 ** 30], p[0, vocab - 1] = 0.5, 0.125, 0.25, 0.125
    q = torch.zeros(1, vocab, dtype=torch.bfloat16, device=DEV) if given else None
    if given:
        q[0, 5] = 1.0
    for sample, token in ((0.1, 77), (0.25, 2 ** 30), (0.7, 2 ** 30), (0.9, vocab - 1)):      # of 1/8, 1/4 and 1/8
        path, count, following = verify("bf16", p.expand(2, vocab), q.expand(2, vocab) if given else None, [0, 5], [-1, 0],
                                        [0, 2], torch.full((2,), 0.75, device=DEV), torch.full((1,), sample, device=DEV), 2)
        assert path.tolist() == [[0, -1]] and count.tolist() == [1] and following.tolist() == [token]


@ALL
@pytest.mark.parametrize("given", [True, False])
def test_verify_edges(typ, given):
    """Random numbers at their ends, tokens and parents out of range, the same token twice, probabilities that are 0,
    negative, infinite or NaN, rows with nothing left."""
    vocab, drafts = 300, [12, 12, 12, 4, 4, 1]
    rng = np.random.default_rng(4)
    parents = [[-1] + [int(rng.integers(0, j)) for j in range(1, 12)] for _ in range(3)] + [[-1, 0, 0, 0]] * 2 + [[-1]]
    parents[1] = [-1, 0, 5, 2, 3, -1, 99, 0, 1, 7, 9, 1 << 30]
    n = sum(drafts)
    p, q = spread(n, vocab, typ, 9, 0.3)
    tokens = drawn(q, parents, drafts, 3)
    tokens[14], tokens[15], tokens[19] = -1, vocab, 1 << 30
    tokens[25:29] = [tokens[24]] * 4
    p[24, 50:] = 0.0                                       # the third sequence's first row: a few tokens are left
    p[0, 10], p[0, 11], p[0, 12], q[0, 13] = math.nan, math.inf, -0.5, math.nan
    p[36], q[36] = 0.0, 1.0 / vocab                        # nothing to draw from
    p[40] = q[40]                                          # nothing left once a draft falls
    tokens[41:44] = [5, 5, 6]
    for accept in (torch.zeros(n, device=DEV), torch.full((n,), 1 - 2.0 ** -24, device=DEV), uniform(n, 1)):
        for sample in (torch.zeros(6, device=DEV), torch.full((6,), 1 - 2.0 ** -24, device=DEV), uniform(6, 2),
                       torch.full((6,), 1.5, device=DEV), torch.full((6,), -1.0, device=DEV)):
            check_verify(typ, p, q if given else None, tokens, parents, drafts, accept, sample)
    check_verify(typ, p, q if given else None, tokens, parents, drafts, uniform(n, 5), uniform(6, 6), most=5)
    # offsets that are clipped or descend, rows before the first sequence
    flat = [x for t in parents for x in t]
    path, count, following = verify(typ, p, q if given else None, tokens, flat, [40, 36, 1000000, -4], uniform(n, 1),
                                    uniform(3, 1), 12)
    assert count[0] == 0 and following[0] == -1 and (path[0] == -1).all() and count[2] == 0
    assert count[1] >= 1 and path[1, 0] == 36


def test_verify_keeps_the_models_distribution():
    """The token behind the root, accepted or drawn anew, is distributed as p: 65000 sequences with siblings drawn from
    a q that is far from it; every frequency within 5 standard deviations."""
    vocab, n, m = 6, 65000, 4
    p1, q1 = torch.tensor([0.02, 0.4, 0.05, 0.3, 0.13, 0.1]), torch.tensor([0.5, 0.05, 0.1, 0.1, 0.2, 0.05])
    p, q = (x.to(DEV).expand(n * m, vocab) for x in (p1, q1))
    tokens = torch.multinomial(q1, n * m, True, generator=torch.Generator().manual_seed(1))
    parent = [-1, 0, 0, 0] * n
    for given in (True, False):
        path, count, following = verify("f32", p, q if given else None, tokens.tolist(), parent, [m * i for i in range(n + 1)],
                                        uniform(n * m, 2), uniform(n, 3), m)
        assert int(count.min()) == 1 and int(count.max()) == 2
        second = torch.where(count == 2, tokens.to(DEV)[path[:, 1].clamp(min=0).long()].int(), following).cpu()
        got = torch.bincount(second.long(), minlength=vocab).double() / n
        if given:
            assert ((got - p1.double()).abs() <= 5 * torch.sqrt(p1 * (1 - p1) / n).double() + 1e-6).all(), got
        assert 0.2 < float((count == 2).float().mean()) < 0.98


@pytest.mark.parametrize("tokens", ["fixed", "any"])
def test_verify_certain_drafts_keep_the_models_distribution(tokens):
    """The same without draft probabilities: whatever the drafted tokens are, the one that comes out is distributed as p."""
    vocab, n, m = 6, 65000, 4
    p1 = torch.tensor([0.02, 0.4, 0.05, 0.3, 0.13, 0.1])
    p = p1.to(DEV).expand(n * m, vocab)
    if tokens == "fixed":
        drafts = torch.tensor([0, 1, 4, 3]).repeat(n)
    else:                                              # a token twice among them
        drafts = torch.randint(0, vocab, (n * m,), generator=torch.Generator().manual_seed(1))
    path, count, following = verify("f32", p, None, drafts.tolist(), [-1, 0, 0, 0] * n, [m * i for i in range(n + 1)],
                                    uniform(n * m, 2), uniform(n, 3), m)
    assert int(count.min()) == 1 and int(count.max()) == 2
    second = torch.where(count == 2, drafts.to(DEV)[path[:, 1].clamp(min=0).long()].int(), following).cpu()
    got = torch.bincount(second.long(), minlength=vocab).double() / n
    assert ((got - p1.double()).abs() <= 5 * torch.sqrt(p1 * (1 - p1) / n).double() + 1e-6).all(), got
    stood = float((count == 2).float().mean())
    if tokens == "fixed":                              # 0.4 + 0.13 + 0.3
        assert abs(stood - 0.83) <= 5 * math.sqrt(0.83 * 0.17 / n)


# ---------------------------------------------------------------- together

def step_inputs(seed, n, heads, kv, dim, vocab, dt):
    q, k, v = randn((n, heads, dim), dt, seed), randn((n, kv, dim), dt, seed + 1), randn((n, kv, dim), dt, seed + 2)
    p, qq = spread(n, vocab, "f32", seed)
    return dict(q=q, k=k, v=v, p=p, qq=qq, accept=uniform(n, seed), sample=uniform(2, seed + 5),
                tokens=torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(seed)).int().to(DEV),
                pos=i32([seed % 50 + j for j in range(n)]))


def test_step_in_a_graph():
    """Rotation, attention of the drafts, their check, room in the cache and the accepted ones kept, recorded once and
    replayed on other inputs and lengths with eager work between: every replay leaves what the eager step leaves.  Two
    recorded graphs share the workspaces."""
    heads, kv, dim, vocab, drafts = 4, 2, 64, 5003, [7, 5]
    n, dt = sum(drafts), torch.bfloat16
    caches = []
    for _ in range(2):
        c = Cache(kv, dim, 32, 80, 2, 40, layers=2)
        k, v = randn((900, kv, dim), dt, 1), randn((900, kv, dim), dt, 2)
        for s in (0, 1):
            c.reserve([s], [450])
            for layer in range(2):
                c.append(k[450 * s:450 * s + 450], v[450 * s:450 * s + 450], [s], [450], "bf16", layer)
        caches.append(c)
    parent, cu, seqs = i32([-1, 0, 0, 1, 1, 2, 4] + [-1, 0, 1, 2, 3]), i32(offsets(drafts)), i32([1, 0])
    d = desc("bf16", heads, kv, dim, 2, 0, 1280)
    size, r = I.ios_attn_tree_work_bytes(d, n, 7), rotary(dim)
    assert size > 0
    dv = I.ios_verify_desc(I.IOS_F32, 2, vocab, 7)
    vsize = I.ios_verify_work_bytes(dv)
    work, vwork = (torch.full((max(x, 16),), 255, dtype=torch.uint8, device=DEV) for x in (size, vsize))
    x = step_inputs(0, n, heads, kv, dim, vocab, dt)
    rows = lambda t: I.ios_rows(t.data_ptr(), t.shape[0], t.stride(0))  # noqa: E731
    outs = [dict(q=torch.zeros_like(x["q"]), k=torch.zeros_like(x["k"]), o=torch.zeros_like(x["q"]),
                 path=torch.zeros(2, 7, dtype=torch.int32, device=DEV), count=i32([0, 0]), next=i32([0, 0])) for _ in range(2)]

    def step(c, y):
        s = stream()
        I.ios_rotate(r, I.IOS_BF16, dim, toks(x["q"]), toks(y["q"]), heads, toks(x["k"]), toks(y["k"]), kv,
                     x["pos"].data_ptr(), s)
        for layer in range(2):
            I.ios_attn_tree(c.c, layer, d, toks(y["q"]), toks(y["k"]), toks(x["v"]), toks(y["o"]), 0, seqs.data_ptr(),
                            cu.data_ptr(), parent.data_ptr(), 7, work.data_ptr(), size, s)
        I.ios_verify(dv, rows(x["p"]), rows(x["qq"]), x["tokens"].data_ptr(), parent.data_ptr(), cu.data_ptr(),
                     x["accept"].data_ptr(), x["sample"].data_ptr(), y["path"].data_ptr(), y["count"].data_ptr(),
                     y["next"].data_ptr(), vwork.data_ptr(), vsize, s)
        I.ios_cache_reserve(c.c, 2, seqs.data_ptr(), y["count"].data_ptr(), s)
        for layer in range(2):
            I.ios_cache_keep(c.c, layer, I.IOS_BF16, toks(y["k"]), toks(x["v"]), 2, seqs.data_ptr(), y["path"].data_ptr(), 7,
                             y["count"].data_ptr(), s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                       # a stream of its own
        step(caches[0], outs[0])
    torch.cuda.current_stream().wait_stream(side)
    step(caches[1], outs[1])
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(caches[0], outs[0])
        graphs.append(g)
    for i in range(9):
        for name, t in step_inputs(17 * i + 3, n, heads, kv, dim, vocab, dt).items():
            x[name].copy_(t)
        for t in outs[0].values():
            t.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        step(caches[1], outs[1])
        torch.cuda.synchronize()
        assert caches[0].lens.tolist() == caches[1].lens.tolist()
        for name in outs[0]:
            assert torch.equal(outs[0][name], outs[1][name]), (i, name)
        for layer in range(2):
            for s, m in enumerate(caches[0].lens.tolist()):
                a, b = (c.read([s], [m], layer=layer) for c in caches)
                assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
                # what was kept last is what stood
                row = [1, 0].index(s)
                kept = outs[0]["path"][row, :int(outs[0]["count"][row])].long()
                assert equal(a[0][m - len(kept):], held(outs[0]["k"][kept])) and equal(a[1][m - len(kept):], held(x["v"][kept]))
    assert I.ios_cache_status(caches[0].c, stream()) == 0


def test_example_drafts():
    """The example's path, end to end: what stood is what the cache grew by, and the same comes out again."""
    import importlib.util
    import os
    import sys
    folder = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
    spec = importlib.util.spec_from_file_location("draft_answers", os.path.join(folder, "draft_answers.py"))
    ex = importlib.util.module_from_spec(spec)
    before = list(sys.path)
    try:
        spec.loader.exec_module(ex)
    finally:
        sys.path[:] = before
    ids, stood, dec = ex.answers(3, 6)
    assert len(stood) == 6 and all(1 <= x <= 4 for row in stood for x in row)
    counts = [sum(row[i] for row in stood) for i in range(3)]
    assert [len(r) for r in ids] == counts and len({r[0] for r in ids}) == 3
    assert all(0 <= t < ex.VOCAB for r in ids for t in r)
    assert dec.lens.tolist() == [1225] + [1225 + m for m in counts]
    again = ex.answers(3, 6)
    assert again[0] == ids and again[1] == stood
