"""The decoder operators at the ends of the numbers' range: weights, scales and
values that are finite or infinite by the definition and must be so in the
result, wherever in a sequence they stand.

Helpers and the bounds of ordinary results are those of test_gpu_decoder."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_decoder import DEV, TYPES, Cache, I, check_prompt, i32, prompt, randn          # noqa: E402

ALL = pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])


def scored(scores, typ, dim=32):
    """Keys whose score with a query of one in the first place is `scores` (scale 1)."""
    k = torch.zeros(len(scores), 1, dim, dtype=TYPES[typ][0], device=DEV)
    k[:, 0, 0] = torch.as_tensor(scores).to(k)
    return k


def one_query(rows, typ, dim=32):
    q = torch.zeros(rows, 1, dim, dtype=TYPES[typ][0], device=DEV)
    q[:, :, 0] = 1.0
    return q


@pytest.mark.parametrize("rows", [1, 200])
@pytest.mark.parametrize("work", [True, False])
def test_prompt_large_values_float32(rows, work):
    """Values of 1e35 whose largest weights come after smaller ones: the sum of 256 weights of at most 1 times 1e35
    stays in float32's range."""
    k = scored([0.0] * 64 + [4.8] * 256, "f32")
    v = torch.full((320, 1, 32), 1e35, device=DEV)
    v[::3] *= -1
    check_prompt("f32", one_query(rows, "f32"), k, v, [rows], [320], 0, 1.0, work=work)
    long = scored([0.0] * 1200 + [4.8] * 256, "f32")
    v = torch.full((1456, 1, 32), 1e34, device=DEV)
    check_prompt("f32", one_query(rows, "f32"), long, v, [rows], [1456], 0, 1.0, work=work)


@pytest.mark.parametrize("n", [71, 1100])
@pytest.mark.parametrize("rows", [1, 200])
@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_prompt_values_near_the_largest(typ, rows, n):
    """Two keys count, the second ahead of the first by 1.3 (1.9 powers of two), both with values of 2e38."""
    s = [-90.0] * n
    s[0], s[70] = 0.0, 1.3
    v = torch.full((n, 1, 32), 2e38, device=DEV).to(TYPES[typ][0])
    check_prompt(typ, one_query(rows, typ), scored(s, typ), v, [rows], [n], 0, 1.0, work=False)


@ALL
def test_prompt_one_key_of_the_largest_value(typ):
    dt = TYPES[typ][0]
    big = torch.finfo(dt).max / (2 if typ == "f32" else 1)
    v = torch.full((3, 2, 64), big, dtype=dt, device=DEV)
    v[1] *= -1
    q, k = randn((3, 2, 64), dt, 1), randn((3, 2, 64), dt, 2)
    check_prompt(typ, q, k, v, [1, 1, 1], [1, 1, 1], 1)


@pytest.mark.parametrize("n", [300, 1300])
@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_prompt_rows_beside_large_values(typ, n):
    """Sums that leave float32's range before they are divided change no row that does not see their keys."""
    dt = TYPES[typ][0]
    q, k, v = randn((n, 2, 64), dt, 1), randn((n, 1, 64), dt, 2), randn((n, 1, 64), dt, 3)
    ref = check_prompt(typ, q, k, v, [n], [n], 1, work=False)
    v[n - 50:] = 3e38
    out = check_prompt(typ, q, k, v, [n], [n], 1, work=False)
    assert torch.equal(out[:n - 50], ref[:n - 50]) and torch.isfinite(out).all()


@pytest.mark.parametrize("scale", [0.0, 1e-35, -1e-35, 1e-40])
@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_prompt_small_scales_of_large_scores(typ, scale):
    """Products of queries and keys up to 1e37: a scale of 0 weighs every key alike, a small one as it says."""
    dt, n = TYPES[typ][0], 200
    size = {0.0: 1e17, 1e-35: 1e17, -1e-35: 1e17, 1e-40: 1e18}[scale]
    q, k = randn((n, 2, 64), dt, 1, size), randn((n, 2, 64), dt, 2, size)
    check_prompt(typ, q, k, randn((n, 2, 64), dt, 3), [n], [n], 1, scale)
    check_prompt(typ, q, k, randn((n, 2, 64), dt, 3), [n], [n], 0, scale)


@ALL
@pytest.mark.parametrize("rows,n,work", [(300, 300, False), (1300, 1300, False), (3, 1300, True), (3, 1300, False),
                                         (70, 6000, True)])
@pytest.mark.parametrize("lead", [0.0, 60.0, 120.0])
def test_prompt_seen_infinities(typ, rows, n, work, lead):
    """An infinite value that a row sees is infinite in its result, however little its key weighs and wherever the key
    lies: in tiles that every row sees or not, before keys far ahead of it or after."""
    s = [0.0] * n
    first = n - rows + 1                          # keys that every row sees
    where = [5, 70, 140, n // 2, n - 2]
    for i in where:
        s[i] = -lead
    s[first // 2] = lead                          # far ahead of all
    v = randn((n, 1, 32), TYPES[typ][0], 3)
    for d, i in enumerate(where):
        v[i, 0, d] = math.inf if d % 2 else -math.inf
        v[i, 0, 8] = math.inf
        v[i, 0, 9] = math.inf if d < 3 else -math.inf
        v[i, 0, 10 + d] = math.nan
    check_prompt(typ, one_query(rows, typ), scored(s, typ), v, [rows], [n], 1, 1.0, work=work)
    check_prompt(typ, one_query(rows, typ), scored(s, typ), v, [rows], [n], 0, 1.0, work=work)


@pytest.mark.parametrize("n,work", [(200, False), (1300, False), (3000, True)])
@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_prompt_scores_beyond_float32_are_not_zeros(typ, n, work):
    """Where scores times log2(e) leave float32's range there is no result; it reads as NaN, not as a row of zeros."""
    dt = TYPES[typ][0]
    q, k = (torch.full((3 if x else n, 1, 32), 2.5e18, dtype=dt, device=DEV) for x in (1, 0))   # scores of 3e38
    k[1::2] *= 0.5
    out, lse, _ = prompt(typ, q, k, randn((n, 1, 32), dt, 3), [3], [n], 0, 1.5, work)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


def test_status_stays_on_its_stream():
    """The flags are cleared on the caller's stream, so before whatever it is given next, and without waiting for the
    default stream: that is still at work when the calls return."""
    c = Cache(1, 32, 32, 2, 2, 4)
    seq, add = i32([0]), i32([100])               # more than there are pages for
    mine = torch.cuda.Stream()
    a = torch.zeros(8192, 8192, dtype=torch.bfloat16, device=DEV)
    b = torch.empty_like(a)
    torch.mm(a, a, out=b)
    torch.cuda.synchronize()
    seen = []
    for _ in range(200):                          # about 1 ms each
        torch.mm(a, a, out=b)
    for _ in range(3):
        I.ios_cache_reserve(c.c, 1, seq.data_ptr(), add.data_ptr(), mine.cuda_stream)
        seen += [I.ios_cache_status(c.c, mine.cuda_stream), I.ios_cache_status(c.c, mine.cuda_stream)]
    busy = not torch.cuda.default_stream().query()
    torch.cuda.synchronize()
    assert seen == [I.IOS_CACHE_NO_PAGES, 0] * 3
    assert busy


@ALL
@pytest.mark.parametrize("rows,n,work", [(1, 7, False), (200, 200, False), (300, 1300, False), (40, 3000, True)])
@pytest.mark.parametrize("dim", [64, 128])
def test_prompt_values_of_the_largest_number(typ, rows, n, work, dim):
    """A mean of the type's largest number is that number, not infinity, whatever the weights' rounding."""
    dt = TYPES[typ][0]
    q, k = randn((rows, 2, dim), dt, 1), randn((n, 1, dim), dt, 2)
    big = torch.finfo(dt).max
    v = torch.full((n, 1, dim), big, dtype=dt, device=DEV)
    v[:, :, 1::2] *= -1
    v[n // 2:, 0, 5] = math.inf                    # which some rows see
    out, _, _ = prompt(typ, q, k, v, [rows], [n], 1, None, work)
    out, u = out.double().cpu(), TYPES[typ][2]
    seen = torch.arange(rows) + n - rows >= n // 2
    assert (out[seen][:, :, 5] == math.inf).all()
    out[:, :, 5] = -big
    out[:, :, 1::2] *= -1
    assert torch.isfinite(out).all() and (out >= big * (1 - 4 * u - 2.0 ** -20)).all() and (out <= big).all()


@pytest.mark.parametrize("n,work", [(2000, False), (900, False), (6000, True)])
@pytest.mark.parametrize("typ,step", [("f16", 2.0 ** -11), ("bf16", 2.0 ** -8)])
def test_prompt_weights_that_all_round_up(typ, step, n, work):
    """Weights half a unit of the type above that of the first keys, all rounded up, their sum not."""
    big = torch.finfo(TYPES[typ][0]).max
    v = torch.full((n, 1, 32), big, dtype=TYPES[typ][0], device=DEV)
    out, _, _ = prompt(typ, one_query(1, typ), scored([0.0] * 128 + [step] * (n - 128), typ), v, [1], [n], 0, 1.0, work)
    assert (out == big).all()
