"""Single-token attention over the 4-bit cache with bounds that a wrong result
cannot meet, and the prompt kernels' forms that only long prompts take.

The bound of an element follows what the operator sums, from the cache's own
numbers: a key is z + s c, its score scale (z sum q + s (c . q)), a value's part
of the result p z + (p s) c.  With p the softmax, A = sum p (|z| + 15 s) and u
the relative rounding error of the result's type:

    |o - ref| <= u |ref| + 2^-25 + (2 e + 2^-18) A + w + 2^-24 R (S + |ref|)

e   error of a score: scale max_j sum_d |q_d| (|z| + 15 s) times 2^-22 (queries and
    their sums in two 16-bit parts of 11 bits) + 2^-24 (head_dim + 8) (32-bit sums);
    2^-18 for the exponential's argument (below 40, 24 bits) and its value
w   roundings before the second product: p and the value held to f16 for bf16
    results (2^-10 A, and 2^-38 of the largest value a key for weights below f16's
    range); p s to two bf16 parts times codes of up to 143 for f16 results; to three
    parts times codes of up to 15 for float32
S   what is summed in 32 bits: A; for f16 results sum p (|z| + 271 s), whose codes
    carry an offset of 128 that the zero points take back
R   roundings one behind the other: 33 a tile (its 32 products, one after the other
    at worst, and the sum so far) for the tiles of one wave, 8 waves, 40 for
    rescaling and the last steps, and the parts."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
I = pytest.importorskip("paper_2011_01302_amd")

from test_gpu_decoder import (DEV, TYPES, Cache, attend, causal_mask, check, check_prompt, decode, desc, offsets,  # noqa: E402
                              prompt, randn)

gpu = pytest.mark.gpu
ALL = pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])


def quantised(x):
    """z, s and c [..., d] of what the cache holds for x, from the format's definition, in numpy's float32."""
    x = x.float().cpu().numpy()
    y = np.minimum(np.maximum(x, np.float32(-61440)), np.float32(61440)).reshape(x.shape[:-1] + (-1, 32))
    lo, hi = y.min(-1, keepdims=True), y.max(-1, keepdims=True)
    z = lo.astype(np.float16).astype(np.float32)
    s = ((hi - lo) * np.float32(1.0 / 15.0)).astype(np.float16).astype(np.float32)
    with np.errstate(all="ignore"):
        c = np.where(s > 0, np.clip(np.rint((y - z) / s), 0, 15), 0).astype(np.float32)
    wide = np.zeros_like(y)
    return [torch.from_numpy((a + wide).reshape(x.shape)).double() for a in (z, s, c)]


def tiles_of_a_wave(d, n, work):
    """Tiles that one of a workgroup's eight waves walks, and the number of parts."""
    size = (d.head_dim + 2) * 4 * d.heads * d.seqs
    parts = max(1, I.ios_attn_work_bytes(d, d.seqs) // size) if work else 1
    chunk = -(-(d.max_keys or 1 << 16) // (32 * parts))
    tiles = -(-n // 32)
    return -(-max(min(chunk, tiles), tiles - (parts - 1) * chunk) // 8), parts


def reference(typ, q, k, v, scale, tiles, parts):
    """Rows q [h][d] over the quantised keys and values of one head: result, log-sum-exp, and bounds of both."""
    q, (kz, ks, kc), (vz, vs, vc) = q.double().cpu(), k, v
    s = scale * (q @ (kz + ks * kc).T)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    out = p @ (vz + vs * vc)
    e = abs(scale) * (q.abs() @ (kz.abs() + 15 * ks).T).amax(1, keepdim=True) * (2.0 ** -22 + 2.0 ** -24 * (q.shape[1] + 8))
    a, ps = p @ (vz.abs() + 15 * vs), p @ vs
    w, summed = {"bf16": (2.0 ** -10 * a + 2.0 ** -38 * len(kz) * float((vz + vs * vc).abs().max()), a),
                 "f16": (2.0 ** -16 * 143 * ps, p @ (vz.abs() + 271 * vs)), "f32": (2.0 ** -24 * 15 * ps, a)}[typ]
    r = 33 * tiles + 8 + 40 + parts
    bound = TYPES[typ][2] * out.abs() + 2.0 ** -25 + (2 * e + 2.0 ** -18) * a + w + 2.0 ** -24 * r * (summed + out.abs())
    return out, lse, bound, e[:, 0] + 2.0 ** -18 + 2.0 ** -24 * r + 2.0 ** -22 * (1 + lse.abs())


# dim, page, heads of keys, queries of each, lengths, max_keys (0: unknown)
CASES = [(64, 64, 2, 3, [9000, 2049], 9000), (64, 64, 2, 3, [9000, 2049], 1 << 20), (96, 32, 2, 4, [5000, 1, 1300], 5000),
         (128, 128, 2, 8, [5003], 5003), (128, 32, 1, 4, [5003, 700], 1 << 16), (32, 256, 1, 20, [4097, 777], 0),
         (96, 64, 1, 17, [3333], 100)]


def data(case):
    """Keys and values on the CPU; the values' mean drifts along the sequence, so that no part can be missed."""
    dim, _, kv, _, lens, _ = CASES[case]
    g = torch.Generator().manual_seed(case)
    k, v = (torch.randn(sum(lens), kv, dim, generator=g) for _ in range(2))
    at = torch.cat([torch.linspace(-1.0, 1.0, m) for m in lens])[:, None, None]
    return k, v + at, torch.randn(len(lens), kv * CASES[case][3], dim, generator=g)


@ALL
@pytest.mark.parametrize("work", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_bounds_refuse_wrong_results(typ, case, work):
    """On the CPU: zeros, a part whose sum or whose keys are missing, missing zero points and scales that are one token
    off are outside the bound of the longest sequence."""
    dim, _, kv, ratio, lens, most = CASES[case]
    k, v, q = data(case)
    d = desc(typ, kv * ratio, kv, dim, len(lens), 0, most)
    k, v, q = k[:lens[0], 0], v[:lens[0], 0], q[0, :ratio].to(TYPES[typ][0])
    kq, vq = quantised(k), quantised(v)
    tiles, parts = tiles_of_a_wave(d, lens[0], work)
    out, lse, bound, far = reference(typ, q, kq, vq, d.scale, tiles, parts)

    def refused(x):
        return bool(((x - out).abs() > bound).any())
    s = d.scale * (q.double() @ (kq[0] + kq[1] * kq[2]).T)
    p = torch.softmax(s, 1)
    kept = torch.ones(lens[0], dtype=torch.float64)
    kept[:min(lens[0] // 4, 256)] = 0.0                      # 256 keys: the smallest part there is
    values = vq[0] + vq[1] * vq[2]
    assert refused(torch.zeros_like(out))
    assert refused((p * kept) @ values)
    assert refused((p * kept) @ values / (p * kept).sum(1, keepdim=True))
    assert refused(p @ (vq[1] * vq[2]))
    assert refused(p @ (vq[0] + vq[1].roll(1, 0) * vq[2]))
    assert (lse - torch.log((torch.exp(s) * kept).sum(1))).abs().max() > far.max()


@gpu
@ALL
@pytest.mark.parametrize("work", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_decode_within_bounds(typ, case, work):
    print("\n[gpu-case] decode", typ, CASES[case], work, flush=True)
    dim, page, kv, ratio, lens, most = CASES[case]
    k, v, q = data(case)
    c = Cache(kv, dim, page, 400, len(lens), 300)
    c.place(lens, case)
    c.append(k.to(DEV), v.to(DEV), list(range(len(lens))), lens, "f32")
    q = q.to(TYPES[typ][0]).to(DEV)
    out, lse, scale = decode(c, typ, q, list(range(len(lens))), most, work)
    d, o = desc(typ, kv * ratio, kv, dim, len(lens), 0, most), offsets(lens)
    for i, m in enumerate(lens):
        tiles, parts = tiles_of_a_wave(d, m, work)
        for h in range(kv):
            rows = slice(h * ratio, (h + 1) * ratio)
            ref, l64, bound, far = reference(typ, q[i, rows], quantised(k[o[i]:o[i + 1], h]), quantised(v[o[i]:o[i + 1], h]),
                                             scale, tiles, parts)
            err = (out[i, rows].double().cpu() - ref).abs()
            assert (err <= bound).all(), (i, h, float((err / bound).max()))
            assert ((lse[rows, i].double().cpu() - l64).abs() <= far).all()


def tail(n):
    """One key 18 ahead of n - 1 equal ones, whose weights of 2^-26 count by their number and their values."""
    k, v = torch.zeros(n, 32), torch.full((n, 32), 1000.0)
    k[77, 0], v[77] = 18.0, -1.0
    q = torch.zeros(1, 32)
    q[:, 0] = 1.0
    return k, v, q


@ALL
@pytest.mark.parametrize("work", [True, False])
def test_bounds_refuse_a_lost_tail(typ, work):
    n = 50000
    k, v, q = tail(n)
    out, lse, bound, far = reference(typ, q.to(TYPES[typ][0]), quantised(k), quantised(v), 1.0,
                                     *tiles_of_a_wave(desc(typ, 1, 1, 32, 1, 0, n, 1.0), n, work))
    assert ((out + 1.0).abs() > bound).all() and (lse - 18.003).abs().item() < 0.01
    top = float((quantised(k)[0] + quantised(k)[1] * quantised(k)[2])[77, 0])
    assert (lse - top).abs().item() > far.item()


@gpu
@ALL
@pytest.mark.parametrize("work", [True, False])
def test_decode_long_tail_counts(typ, work):
    n = 50000
    k, v, q = tail(n)
    c = Cache(1, 32, 256, 200, 1, 200)
    c.place([n])
    c.append(k[:, None].to(DEV), v[:, None].to(DEV), [0], [n], "f32")
    q = q[None].to(TYPES[typ][0]).to(DEV)
    out, lse, _ = decode(c, typ, q, [0], n, work, scale=1.0)
    ref, l64, bound, far = reference(typ, q[0], quantised(k), quantised(v), 1.0,
                                     *tiles_of_a_wave(desc(typ, 1, 1, 32, 1, 0, n, 1.0), n, work))
    assert ((out[0].double().cpu() - ref).abs() <= bound).all()
    assert abs(float(lse) - float(l64)) <= float(far)


# ---------------------------------------------------------------- prompts of 1024 keys and more

@gpu
@ALL
@pytest.mark.parametrize("dim", [32, 40, 64, 96, 128])
@pytest.mark.parametrize("work", [True, False])
def test_prompt_long_head_dims(typ, dim, work):
    """Two groups of waves, or the keys in parts, for every head size; whole tiles of queries, and rows past the keys."""
    dt = TYPES[typ][0]
    for lq, lk, causal in (([1100], [1100], 1), ([1537, 130], [1537, 1410], 1), ([200], [2111], 0), ([1200], [1030], 1)):
        q = randn((sum(lq), 2, dim), dt, 1)
        k, v = randn((sum(lk), 1, dim), dt, 2), randn((sum(lk), 1, dim), dt, 3)
        check_prompt(typ, q, k, v, lq, lk, causal, what="long", work=work)


@gpu
@ALL
@pytest.mark.parametrize("dim", [32, 40, 96, 128])
@pytest.mark.parametrize("rows,n,work", [(300, 300, False), (1300, 1300, False), (40, 3000, True)])
def test_prompt_infinities_and_nan_in_every_form(typ, dim, rows, n, work):
    """What a row sees reaches it, what it does not see leaves it as it was, to the bit: one workgroup, two groups of
    waves and parts, for every head size."""
    dt = TYPES[typ][0]
    q, k, v = randn((rows, 2, dim), dt, 7), randn((n, 1, dim), dt, 8), randn((n, 1, dim), dt, 9)
    ref, lse0, _ = prompt(typ, q, k, v, [rows], [n], 1, None, work)
    cut = rows - rows // 4                                   # the first row that sees the keys from here on
    odd = n - rows + cut
    v[odd:, 0, 3], v[odd + 1:, 0, 5], v[odd + 2:, 0, 5], v[odd:, 0, dim - 1] = math.nan, math.inf, -math.inf, math.inf
    check_prompt(typ, q, k, v, [rows], [n], 1, work=work)
    out, lse, _ = prompt(typ, q, k, v, [rows], [n], 1, None, work)
    assert torch.equal(out[:cut], ref[:cut]) and torch.equal(lse, lse0)
    k[odd] = math.nan
    out, lse, _ = prompt(typ, q, k, v, [rows], [n], 1, None, work)
    assert torch.equal(out[:cut], ref[:cut]) and torch.equal(lse[:, :cut], lse0[:, :cut])
    assert torch.isnan(out[cut:]).all()


@gpu
@ALL
@pytest.mark.parametrize("most", [1, 700, 1 << 20])
def test_prompt_max_keys_only_costs_speed(typ, most):
    """max_keys far below or above the lengths, as a recorded call that knows only its capacity gives it."""
    dt, lq, lk, dim = TYPES[typ][0], [1, 40, 0, 131], [5000, 40, 3, 700], 64
    q, k, v = (randn((sum(x), h, dim), dt, s) for x, h, s in ((lq, 4, 1), (lk, 2, 2), (lk, 2, 3)))
    d = desc(typ, 4, 2, dim, len(lq), 1, most)
    size = I.ios_attn_work_bytes(d, q.shape[0])
    work = torch.full((max(size, 16),), 255, dtype=torch.uint8, device=DEV)
    out, oq, ok = torch.zeros_like(q), offsets(lq), offsets(lk)
    cu_q, cu_k = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (oq, ok))
    t = [I.ios_tokens(x.data_ptr(), x.shape[0], x.stride(0), x.stride(1)) for x in (q, k, v, out)]
    I.ios_attn_prompt(d, *t, 0, cu_q.data_ptr(), cu_k.data_ptr(), work.data_ptr(), size, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    u = TYPES[typ][2]
    for i in range(len(lq)):
        for h in range(4):
            ref, a, _, g = attend(q[oq[i]:oq[i + 1], h], k[ok[i]:ok[i + 1], h // 2], v[ok[i]:ok[i + 1], h // 2], d.scale,
                                  causal_mask(lq[i], lk[i], 1))
            check(out[oq[i]:oq[i + 1], h], ref, a, g, u, 0.0 if typ == "f32" else u, lk[i], what=(i, h))


@gpu
@ALL
def test_decode_over_forked_sequences(typ):
    """Answers that share a prompt's pages attend over it and over their own tokens."""
    dim, n = 64, 1234
    k, v, q = randn((n, 2, dim), torch.float32, 1), randn((n, 2, dim), torch.float32, 2), randn((4, 6, dim), TYPES[typ][0], 3)
    c = Cache(2, dim, 32, 80, 4, 50)
    c.reserve([0], [n])
    c.append(k, v, [0], [n], "f32")
    a, b = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 0, 0], [1, 2, 3]))
    I.ios_cache_fork(c.c, 3, a.data_ptr(), b.data_ptr(), torch.cuda.current_stream().cuda_stream)
    x, y = randn((4, 2, dim), torch.float32, 4, 3.0), randn((4, 2, dim), torch.float32, 5, 3.0)
    c.reserve([0, 1, 2, 3], [1] * 4)
    assert I.ios_cache_status(c.c, torch.cuda.current_stream().cuda_stream) == 0
    c.append(x, y, [0, 1, 2, 3], [1] * 4, "f32")
    out, lse, scale = decode(c, typ, q, [0, 1, 2, 3], 1600)
    tiles, parts = tiles_of_a_wave(desc(typ, 6, 2, dim, 4, 0, 1600), n + 1, True)
    for i in range(4):
        for h in range(2):
            rows = slice(3 * h, 3 * h + 3)
            kk, vv = torch.cat([k[:, h], x[i:i + 1, h]]), torch.cat([v[:, h], y[i:i + 1, h]])
            ref, l64, bound, far = reference(typ, q[i, rows], quantised(kk), quantised(vv), scale, tiles, parts)
            assert ((out[i, rows].double().cpu() - ref).abs() <= bound).all()
            assert ((lse[rows, i].double().cpu() - l64).abs() <= far).all()
