"""Rows in 8 bits (quantised, read back, multiplied) and the draw of a class from logits against their definitions in 64 bits.

Integers, scales and tokens are equal.  Tolerances are sums of the roundings on the way (u = 2^-24, a rounding to fp32; half a step of bf16 is 2^-8 of the
value), derived beside each comparison.  Outputs lie in front of canary bytes.
"""
import numpy as np
import pytest
import torch

from paper_2209_13443_b200 import binding as eb
from tests.test_gpu_operators import HALF, TD, U, gen, moved, normal, out_like, untouched

pytestmark = pytest.mark.gpu


def uniform(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def pitch(c):
    return (c + 15) // 16 * 16


# ----------------------------------------------------------------------------- rows in 8 bits

def integers(x):
    """The definition: (integers as fp64, scales as fp32)."""
    big = x.double().abs().amax(1)
    scale = x.float().abs().amax(1) * torch.full((), 1 / 127, dtype=torch.float32, device="cuda")
    bad = ~torch.isfinite(big)
    s = scale.double()[:, None]
    ratio = torch.where((s > 0) & ~bad[:, None], x.double() / s, torch.zeros_like(s))
    low = torch.floor(ratio)
    rest = ratio - low
    q = (low + ((rest > 0.5) | ((rest == 0.5) & (torch.remainder(low, 2) == 1))).double()).clamp(-127, 127)
    return q, torch.where(bad, torch.full_like(scale, float("nan")), scale)


def quantised(x, dtype):
    rows, c = x.shape
    q, raw = out_like((rows, pitch(c)), torch.int8)
    scale, raw_s = out_like((rows,), torch.float32)
    eb.quantize_rows(dtype, x, rows, c, q, scale)
    assert untouched(raw, 0, rows * pitch(c)) and untouched(raw_s, 0, rows)
    return q, scale


def check_rows(x, q, scale):
    want, s = integers(x)
    c = x.shape[1]
    assert torch.equal(scale.view(torch.int32)[~s.isnan()], s.view(torch.int32)[~s.isnan()]) and bool(scale[s.isnan()].isnan().all())
    assert torch.equal(q[:, :c].double(), want) and bool((q[:, c:] == 0).all())


ROWS = [(1, 1), (3, 2), (5, 7), (2, 15), (7, 16), (9, 17), (4, 96), (33, 99), (13, 512), (6, 513), (3, 1000), (5, 1023), (4, 1024), (130, 1026), (2, 4096), (3, 4100), (2, 5001), (2, 16384), (1, 16390), (2, 33001),
        (1, 131071), (1001, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", ROWS)
def test_quantise_and_read_back(rows, c, dtype):
    g = gen(rows + c)
    x = (normal(g, rows, c) * (0.5 + normal(g, c).abs()) + 0.5 * normal(g, c)).to(TD[dtype])
    x[rows // 2] = 0
    q, scale = quantised(x, dtype)
    check_rows(x, q, scale)
    for index in (None, torch.randint(0, rows, (2 * rows + 1,), generator=g, device="cuda").int()):
        count = rows if index is None else 2 * rows + 1
        y, raw = out_like((count, c), TD[dtype])
        eb.dequantize_rows(dtype, q, scale, rows, c, y, count, index=index)
        at = torch.arange(rows, device="cuda") if index is None else index.long()
        ref = q[at, :c].double() * scale[at].double()[:, None]
        # a product rounded to fp32, for bf16 once more
        assert bool(((y.double() - ref).abs() <= ref.abs() * (HALF[dtype] if dtype == "f32" else (1 + HALF[dtype]) * (1 + U) - 1)).all())
        assert untouched(raw, 0, count * c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 4, 3])
def test_rows_off_a_16_byte_boundary(dtype, shift):
    g = gen(shift)
    for rows, c in ((5, 64), (3, 1001), (2, 2600)):
        x = normal(g, rows, c).to(TD[dtype])
        q, scale = quantised(moved(x, shift), dtype)
        check_rows(x, q, scale)
        y, raw = out_like((rows, c), TD[dtype], shift)
        eb.dequantize_rows(dtype, q, scale, rows, c, y, rows)
        aligned, _ = out_like((rows, c), TD[dtype])
        eb.dequantize_rows(dtype, q, scale, rows, c, aligned, rows)
        assert torch.equal(y, aligned) and untouched(raw, shift, rows * c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_middle_of_two_integers_goes_to_the_even_one(dtype):
    """With the largest magnitude 127 * 2^e the scale is 2^e (127 times the float nearest to 1 / 127 rounds to 1): quotients are exact, and every half occurs."""
    half = torch.arange(-253, 254, device="cuda").float() / 2
    rows = torch.stack([torch.cat([half, half.new_tensor([127.0])]) * 2.0 ** e for e in (0, -3, 40, -100, 100)]).to(TD[dtype])
    q, scale = quantised(rows, dtype)
    check_rows(rows, q, scale)
    assert scale.tolist() == [2.0 ** e for e in (0, -3, 40, -100, 100)]
    assert torch.equal(q[0, :507].float(), torch.round(half))
    # next to the middle: the quotient misses it by as little as two floats can
    g = gen(1)
    big = 1 + uniform(g, 400)
    s = big * torch.full((), 1 / 127, dtype=torch.float32, device="cuda")
    x = ((torch.randint(-126, 126, (400, 200), generator=g, device="cuda").double() + 0.5) * s.double()[:, None]).float()
    x = torch.cat([x, torch.nextafter(x, x.new_full((), 9.0)), torch.nextafter(x, x.new_full((), -9.0)), big[:, None]], 1)
    check_rows(x, *quantised(x, "f32"))


def test_every_quotient_of_bf16():
    """A row for each significand of a maximum, with all values of twelve octaves below it: middles of two integers, and what the rounded scale makes of them."""
    top = (0x3f80 + torch.arange(128, device="cuda")).to(torch.int16)
    below = (0x3f80 - 11 * 128 + torch.arange(12 * 128, device="cuda")).to(torch.int16)
    mag = torch.cat([top[:, None], torch.minimum(below[None].expand(128, -1), top[:, None])], 1)
    for power in (0, 100, -100):
        x = torch.cat([mag.view(torch.bfloat16), -mag.view(torch.bfloat16)], 1).mul(2.0 ** power).contiguous()
        for dtype in ("bf16", "f32"):
            v = x.to(TD[dtype])
            check_rows(v, *quantised(v, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_at_the_ends_of_the_type(dtype):
    big, small = torch.finfo(TD[dtype]).max, 2.0 ** -133
    rows = torch.tensor([[big, -big, big / 254, 0], [small, -small, 3 * small, 0], [50 * small, 200 * small, -190 * small, 100 * small], [1e-36, -1e-37, 3e-38, 5e-39], [-0.0, 0.0, 0.0, 0.0],
                         [float("nan"), 1, 2, 3], [1, float("inf"), 2, 3], [1, 2, float("-inf"), float("nan")], [1e-30, 1e30, -1e30, 4e27]], device="cuda").to(TD[dtype])
    for wide in (rows, torch.cat([rows, torch.zeros(9, 1500, device="cuda", dtype=TD[dtype])], 1)):
        q, scale = quantised(wide, dtype)
        check_rows(wide, q, scale)
    assert scale.isnan().tolist() == [False] * 5 + [True] * 3 + [False]
    y, _ = out_like((9, 4), TD[dtype])
    q, scale = quantised(rows, dtype)
    eb.dequantize_rows(dtype, q, scale, 9, 4, y, 9)
    assert y.isnan().all(1).tolist() == [False] * 5 + [True] * 3 + [False]


def test_the_smallest_floats():
    """Scales below 2^-126 have few bits: x / scale passes 127 and is held there."""
    tiny = torch.arange(0, 600, device="cuda", dtype=torch.int32).view(torch.float32)       # the 600 smallest
    rows = torch.stack([tiny * (torch.arange(600, device="cuda") <= top) for top in (0, 1, 63, 64, 100, 190, 191, 400, 599)])
    check_rows(rows, *quantised(rows, "f32"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_reading_leaves_rows_without_a_source_alone(dtype):
    g = gen(3)
    for c in (8, 33, 4096):
        x = normal(g, 6, c).to(TD[dtype])
        q, scale = quantised(x, dtype)
        index = torch.tensor([5, -1, 0, 6, 0, 2 ** 31 - 1, -2 ** 31, 3], dtype=torch.int32, device="cuda")
        y = torch.full((8, c), 55.0, dtype=TD[dtype], device="cuda")
        eb.dequantize_rows(dtype, q, scale, 6, c, y, 8, index=index)
        whole = torch.empty(6, c, dtype=TD[dtype], device="cuda")
        eb.dequantize_rows(dtype, q, scale, 6, c, whole, 6)
        for t, i in enumerate(index.tolist()):
            assert torch.equal(y[t], whole[i] if 0 <= i < 6 else torch.full_like(y[t], 55.0))


def test_a_pool_beyond_2_31_bytes():
    c, pool = 4096, (1 << 31) // 4096 + 5
    q = torch.zeros((pool, c), dtype=torch.int8, device="cuda")
    scale = torch.ones(pool, device="cuda")
    q[-3:] = torch.arange(-64, 64, device="cuda", dtype=torch.int8).repeat(32)
    y = torch.empty((4, c), dtype=torch.bfloat16, device="cuda")
    eb.dequantize_rows("bf16", q, scale, pool, c, y, 4, index=torch.tensor([pool - 1, 0, pool - 3, pool - 4], dtype=torch.int32, device="cuda"))
    assert torch.equal(y[0].float(), q[-1].float()) and torch.equal(y[2].float(), q[-3].float()) and not bool(y[1].any()) and not bool(y[3].any())
    rows = pool // 2 + 3          # 2^31 bytes of bf16 and more on the way back in
    x = torch.zeros((rows, c), dtype=torch.bfloat16, device="cuda")
    x[-2:] = 3
    eb.quantize_rows("bf16", x, rows, c, q[:rows], scale[:rows])
    assert not bool(q[:rows - 2].any()) and bool((q[rows - 2:rows] == 127).all()) and scale[rows - 3:rows].tolist()[0] == 0


# ----------------------------------------------------------------------------- projection

def padded(q):
    out = torch.full((q.shape[0], pitch(q.shape[1])), 99, dtype=torch.int8, device="cuda")     # what lies behind a row is not read
    out[:, :q.shape[1]] = q
    return out


def linear_case(rows, c, n, dtype, seed=0, bias=True):
    g = gen(seed + rows + 3 * c + 7 * n)
    x = normal(g, rows, c).to(TD[dtype])
    w = torch.randint(-127, 128, (n, c), generator=g, device="cuda").to(torch.int8)
    return x, w, 0.001 + 0.01 * uniform(g, n), normal(g, n) if bias else None


def linear_run(x, w, ws, bias, dtype, x_scale=None, shift=0):
    rows, n = x.shape[0], w.shape[0]
    c = w.shape[1]
    y, raw = out_like((rows, n), TD[dtype], shift)
    room = None
    if x_scale is None:
        need = eb.int8_linear_workspace_bytes(rows, c)
        room = torch.full((need + 256 + 64,), 0x55, dtype=torch.uint8, device="cuda")
    eb.int8_linear(dtype, x, rows, c, padded(w), ws, n, y, workspace=room, x_scale=x_scale, bias=bias)
    assert untouched(raw, shift, rows * n)
    if room is not None:
        assert bool((room[(-room.data_ptr()) % 256 + need:] == 0x55).all())
    return y


def linear_check(y, q, xs, w, ws, bias, dtype):
    """bf16: the sum, its product with one scale and the last step are rounded to fp32 (u each), then to bf16; fp32: one rounding of what fp64 gives (2^-50 for its own)."""
    part = (q.double() @ w.double().t()) * (1.0 if ws is None else ws.double()) * xs.double()[:, None]
    ref = part + (0.0 if bias is None else bias.double())
    own = 2.1 * U * part.abs() if dtype == "bf16" else 2.0 ** -50 * (part.abs() + ref.abs())
    last = U + HALF["bf16"] * (1 + U) if dtype == "bf16" else U
    tol = own + last * (ref.abs() + own) + 2.0 ** -149
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), f"off by {float((err / tol).max()):.3g} tolerances"


LINEARS = [(1, 1, 1), (1, 16, 8), (2, 17, 3), (3, 100, 130), (16, 128, 128), (17, 129, 127), (33, 2043, 1001), (1, 2048, 1000), (1, 4096, 4096), (5, 300, 257), (64, 4096, 512), (65, 1000, 96), (100, 512, 1030),
           (128, 4096, 4096), (129, 640, 4100), (200, 2048, 2048), (300, 96, 6000), (513, 1024, 2050), (1000, 333, 3001), (777, 4096, 1500), (2048, 256, 260), (2500, 130, 2000), (20000, 64, 100), (20000, 64, 10),
           (1, 131071, 20), (3, 60000, 300), (256, 8192, 2600), (1500, 1500, 1500)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,n", LINEARS)
def test_int8_linear(rows, c, n, dtype):
    x, w, ws, bias = linear_case(rows, c, n, dtype, bias=(rows + n) % 3 != 0)
    q, xs = integers(x)
    y = linear_run(x, w, ws, bias, dtype)
    linear_check(y, q, xs, w, ws, bias, dtype)
    # quantised before: the same bits, and a row alone has them too
    assert torch.equal(linear_run(padded(q.to(torch.int8)), w, ws, bias, dtype, x_scale=xs), y)
    at = rows // 2
    assert torch.equal(linear_run(x[at:at + 1].contiguous(), w, ws, bias, dtype), y[at:at + 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(2, 129), (200, 300), (1000, 3000)])
def test_int8_linear_at_the_ends_of_the_integers(dtype, rows, n):
    """Sums of 131071 products of -128 and -128 are the largest there are; scales may be missing, NaN or 0."""
    for c in (131071, 4099) if rows < 1000 else (1283,):
        q = torch.full((rows, c), -128, dtype=torch.int8, device="cuda")
        w = torch.full((n, c), -128, dtype=torch.int8, device="cuda")
        w[1::2] = 127
        q[1] = 127
        xs = torch.ones(rows, device="cuda")
        y = linear_run(padded(q), w, None, None, dtype, x_scale=xs)
        linear_check(y, q.double(), xs, w, None, None, dtype)
    xs[0], xs[1] = float("nan"), 0.0
    ws = torch.ones(n, device="cuda")
    ws[2] = float("nan")
    y = linear_run(padded(q), w, ws, torch.full((n,), 2.5, device="cuda"), dtype, x_scale=xs)
    assert bool(y[0].isnan().all()) and bool(y[:, 2].isnan().all()) and bool((y[1, 3:] == 2.5).all()) and not bool(y[2:, 3:].isnan().any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_int8_linear_rows_that_are_not_finite(dtype):
    x, w, ws, bias = linear_case(40, 500, 200, dtype)
    x[7, 3], x[9, 499], x[11] = float("nan"), float("inf"), 0
    y = linear_run(x, w, ws, bias, dtype)
    assert bool(y[[7, 9]].isnan().all()) and torch.equal(y[11], bias.to(TD[dtype]))
    keep = [t for t in range(40) if t not in (7, 9)]
    q, xs = integers(x)
    linear_check(y[keep], q[keep], xs[keep], w, ws, bias, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_int8_linear_off_a_16_byte_boundary(dtype, shift):
    for rows, c, n in ((5, 200, 130), (600, 200, 2100)):
        x, w, ws, bias = linear_case(rows, c, n, dtype)
        assert torch.equal(linear_run(moved(x, shift), w, ws, bias, dtype, shift=shift), linear_run(x, w, ws, bias, dtype))


# ----------------------------------------------------------------------------- the draw

def sample_exact(x, t, k, p, m, u):
    """(token, probabilities) of one row, as the procedure is told."""
    n = len(x)
    if np.isnan(x).any() or np.isposinf(x).any():
        return -1, np.full(n, np.nan)
    top = x.max()
    if np.isneginf(top):
        return -1, np.zeros(n)
    order = np.argsort(-(x + 0.0), kind="stable")
    z = x[order]
    with np.errstate(over="ignore", invalid="ignore"):
        w = np.exp((z - top) / t) if t > 0 else np.zeros(n)
    w[np.isneginf(z)] = 0.0
    if t > 0:
        count = k if 0 < k < n else n
        if p < 1:
            c = np.concatenate([[0.0], np.cumsum(w[:count])])
            count = min(count, max(1, int((c[:-1] < p * c[-1]).sum())))
        if m > 0:
            count = min(count, max(1, int((w[:count] >= m).sum())))
    else:
        count, w[0] = 1, 1.0
    q = np.zeros(n)
    q[order[:count]] = w[:count]
    cum = np.cumsum(q)
    goal = u * cum[-1] if u > 0 else 0.0
    over = np.nonzero(cum > goal)[0]
    token = over[0] if len(over) else np.nonzero(q)[0][-1]
    return int(token), q / cum[-1]


def sample_run(x, dtype, t=None, k=None, p=None, m=None, u=None, probs=True, shift=0):
    rows, n = x.shape
    tokens, raw_t = out_like((rows,), torch.int32)
    out, raw = out_like((rows, n), torch.float32, shift) if probs else (None, None)
    eb.sample(dtype, x, rows, n, u, tokens, temperature=t, top_k=k, top_p=p, min_p=m, probs=out)
    assert untouched(raw_t, 0, rows) and (not probs or untouched(raw, shift, rows * n))
    return tokens, out


def sample_check(x, dtype, t=None, k=None, p=None, m=None, u=None, shift=0):
    """Probabilities: the exponent off by two roundings of its argument (|z| <= 104 where anything is left in fp32), the power by two units, the quotient by two."""
    rows, n = x.shape
    tokens, out = sample_run(x, dtype, t, k, p, m, u, shift=shift)
    alone, _ = sample_run(x, dtype, t, k, p, m, u, probs=False)
    assert torch.equal(tokens, alone)
    host = x.float().cpu().numpy().astype(np.float64)
    at = lambda v, i, d: d if v is None else float(v[i])  # noqa: E731
    for i in range(rows):
        token, q = sample_exact(host[i], at(t, i, 1.0), int(at(k, i, 0)), at(p, i, 1.0), at(m, i, 0.0), at(u, i, 0.0))
        got = out[i].double().cpu().numpy()
        assert int(tokens[i]) == token, (i, int(tokens[i]), token)
        if np.isnan(q).any():
            assert np.isnan(got).all()
            continue
        with np.errstate(divide="ignore"):
            z = np.where(q > 0, np.abs(np.log(q)), 0.0)
        tol = q * (2 * np.minimum(z + 20, 104) + 6) * U + 2.0 ** -126
        assert (np.abs(got - q) <= tol).all(), (i, float((np.abs(got - q) / tol).max()))
        assert ((got > 0) <= (q > 0)).all()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def f32(v):
    return torch.tensor(v, dtype=torch.float32, device="cuda")


SIZES = [1, 2, 7, 31, 64, 255, 1000, 1025, 4097, 16384, 16385, 32769, 50000, 128001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", SIZES)
def test_sample(n, dtype):
    g = gen(n)
    rows = 24
    x = (3 * normal(g, rows, n)).to(TD[dtype])
    heat = 0.5 + uniform(g, rows)
    k = torch.randint(1, min(n, 100) + 1, (rows,), generator=g, device="cuda").int()
    k[::5] = 0
    p = 0.5 + 0.49 * uniform(g, rows)
    m = 0.1 * uniform(g, rows)
    for i, case in enumerate([dict(), dict(t=heat), dict(k=k), dict(p=p), dict(m=m), dict(t=heat, k=k, p=p), dict(t=heat, p=p, m=m), dict(t=heat, k=k, p=p, m=m)]):
        sample_check(x, dtype, u=uniform(gen(n + i), rows), **case)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [300007, 614400])
def test_sample_of_the_longest_rows(n, dtype):
    g = gen(n)
    x = (3 * normal(g, 4, n)).to(TD[dtype])
    for case in (dict(), dict(k=i32([1, 50, 5000, n - 1])), dict(p=f32([0.3, 0.9, 0.999, 0.999999])), dict(k=i32([40, 400, 40000, 400000]), p=f32([0.9, 0.5, 0.99, 0.7]))):
        sample_check(x, dtype, u=uniform(g, 4), **case)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,spread", [(262144, 4.0), (614400, 3.0), (614400, 4.0)])
def test_sample_of_a_nucleus_that_leaves_out_next_to_nothing(n, spread, dtype):
    """top_p one step below 1: what stays outside is 2^-24 of the total, in classes that weigh down to 10^-13 of it.  Weights are off by 2^-47 of theirs (|z| <= 44 octaves in 53 bits, the
    polynomial), sums in fp64 by chains of 180 additions, 2^-45; whole numbers in which the search counts, half a unit of up to 2^-62 of the total for each of n classes:
    2^-43.7.  So the last class that is kept has less than p (1 + 2^-42) of the total in front of it, and p (1 - 2^-42) at least with it."""
    g = gen(n + int(spread))
    rows = 12
    x = (spread * normal(g, rows, n)).to(TD[dtype])
    k = torch.tensor([0, 5000, 0, n // 2] * 3, dtype=torch.int32, device="cuda")
    p, u = 1 - 2.0 ** -24, uniform(g, rows)
    tokens, out = sample_run(x, dtype, k=k, p=f32([p] * rows), u=u)
    host, got = x.float().cpu().numpy().astype(np.longdouble), out.cpu().numpy()
    for i in range(rows):
        order = np.argsort(-host[i], kind="stable")[:int(k[i]) or n]
        w = np.exp(host[i][order] - host[i][order[0]])
        c = np.concatenate([[np.longdouble(0)], np.cumsum(w)])
        count = int((got[i] > 0).sum())
        assert (got[i][order[:count]] > 0).all()               # the first of the order
        goal, off = p * c[-1], np.longdouble(2.0 ** -42)
        assert c[count - 1] < goal * (1 + off) and c[count] >= goal * (1 - off), (i, count, int((c[:-1] < goal).sum()))
        q = np.zeros(n, np.longdouble)
        q[order[:count]] = w[:count]
        cum = np.cumsum(q)
        assert int(tokens[i]) == int(np.nonzero(cum > np.longdouble(float(u[i])) * cum[-1])[0][0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [16000, 32768, 128001])
def test_sample_of_a_nucleus_that_may_end_in_any_bin(n, dtype):
    """One class has all of the weight but 10^-5, and top_p asks for some of the rest, which lies at the far end of what a kept class may be away from the best: (1 - p) / n of the total."""
    g = gen(n)
    p = 1 - np.array([1e-5, 2e-5, 5e-6, 1e-5])
    far = np.log(n / (1 - p.astype(np.float32)).astype(np.float64))
    x = torch.tensor(-far, device="cuda")[:, None] + torch.tensor([0.8, 0.8, 0.8, 6.0], device="cuda").double()[:, None] * uniform(g, 4, n).double()
    x[torch.arange(4), torch.tensor([0, n // 2, n - 1, 7])] = 0.0
    for off in (0.0, 5.0):
        sample_check((x + off).float().to(TD[dtype]), dtype, p=f32(p.tolist()), u=uniform(g, 4))


@pytest.mark.parametrize("n", [16384, 32768, 262080])
def test_sample_of_weights_that_sums_in_fp32_lose(n):
    """One class of weight 1 for each thread (of a part's words, every 256th is a thread's), and a tail of which each weighs less than half a unit in the last place of that: added to it in fp32 they are lost,
    and the nucleus ends among them, at a quarter, a half and three quarters of what they weigh."""
    g = gen(n)
    per = n // max(1, min(8, n // 16384))
    place = torch.arange(n, device="cuda") % per
    tail = -np.log(2.0) * (24.01 + 0.6 * uniform(g, 3, n))
    x = torch.where((place < 1024) & (place % 4 == 0), torch.zeros_like(tail), tail)
    w = torch.exp(x.double())
    out = 1 - (w * (x == 0)).sum(1) / w.sum(1)
    p = (1 - out * torch.tensor([0.75, 0.5, 0.25], device="cuda")).float()
    assert bool((p < 1).all()) and bool((out > 1e-6).all())
    for u in (uniform(g, 3), f32([1 - 2.0 ** -24] * 3)):
        sample_check(x, "f32", p=p, u=u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5, 700, 20000, 128001])
def test_sample_settings_at_their_ends(n, dtype):
    g = gen(n + 1)
    nan, inf = float("nan"), float("inf")
    heats = [1.0, 0.0, -2.0, nan, inf, 1e-30, 1e30, 0.01, 50.0, 1.0]
    rows = len(heats)
    x = (2 * normal(g, rows, n)).to(TD[dtype])
    for t, k, p, m in ((heats, None, None, None), (heats, [3] * rows, [0.6] * rows, None), (None, [0, 1, 2, n - 1, n, n + 5, -3, -2 ** 31, 2 ** 31 - 1, min(n, 513)], None, None),
                       (None, None, [0.0, -1.0, 1e-9, 1e-45, 0.5, 1 - 2.0 ** -24, 1.0, 2.0, nan, 0.9], None), (None, None, None, [0.0, -1.0, 1e-9, 1e-40, 0.5, 1 - 2.0 ** -24, 1.0, 2.0, nan, inf]),
                       (heats, [n - 1] * rows, [1 - 2.0 ** -24] * rows, [1e-30] * rows)):
        for u in ([0.0] * rows, [1 - 2.0 ** -24] * rows, [0.5, 1.0, 2.0, nan, -1.0, inf, 2.0 ** -30, 0.25, 0.75, 0.999]):
            sample_check(x, dtype, t=None if t is None else f32(t), k=None if k is None else i32(k), p=None if p is None else f32(p), m=None if m is None else f32(m), u=f32(u))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [9, 1000, 40001, 128001])
def test_sample_of_equal_and_masked_logits(n, dtype):
    """Ties by the thousand, rows that are masked but for a few, masks of the type's lowest value, zeros of both signs, rows with nothing and rows that are not finite."""
    g = gen(n + 2)
    low, inf = torch.finfo(TD[dtype]).min, float("inf")
    x = torch.zeros(12, n, device="cuda")
    x[1] = -7.25
    x[2] = torch.randint(0, 3, (n,), generator=g, device="cuda").float()
    x[3] = torch.randint(0, 40, (n,), generator=g, device="cuda").float() / 8 - 3
    x[4] = normal(g, n).masked_fill(uniform(g, n) < 0.9, -inf)
    x[5] = normal(g, n).masked_fill(uniform(g, n) < 0.5, low)
    x[6] = -inf
    x[6, n // 3] = low
    x[7] = -inf
    x[8] = normal(g, n)
    x[8, n - 1] = float("nan")
    x[9] = normal(g, n)
    x[9, 0] = inf
    x[10] = torch.where(uniform(g, n) < 0.5, torch.zeros(n, device="cuda"), torch.full((n,), -0.0, device="cuda"))
    x[11] = low
    x = x.to(TD[dtype])
    rows = 12
    u = uniform(g, rows)
    third = max(2, n // 3)
    for case in (dict(), dict(k=i32([third] * rows)), dict(p=f32([0.37] * rows)), dict(k=i32([third] * rows), p=f32([0.61] * rows)), dict(k=i32([2] * rows)), dict(p=f32([0.9999] * rows), m=f32([0.5] * rows)),
                 dict(t=f32([0.0] * rows)), dict(t=f32([inf] * rows), k=i32([third] * rows), p=f32([0.25] * rows)), dict(k=i32([n - 1] * rows), p=f32([0.75] * rows))):
        sample_check(x, dtype, u=u, **case)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 0.05, 20.0, 1e30])
def test_sample_of_logits_of_any_size(dtype, scale):
    g = gen(8)
    for n in (600, 50001):
        x = (normal(g, 6, n).double() * scale + torch.tensor([0.0, 1.0, -1.0, 30.0, -30.0, 0.0], device="cuda").double()[:, None] * min(scale, 1.0)).float().to(TD[dtype])
        x[5] = -x[5].abs() - x[5].abs().max()              # none above 0, as logarithms of probabilities
        for case in (dict(), dict(k=i32([40] * 6)), dict(p=f32([0.8] * 6)), dict(t=f32([scale] * 6), k=i32([n // 2] * 6), p=f32([0.9] * 6))):
            sample_check(x, dtype, u=uniform(g, 6), **case)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [700, 20000, 128001])
def test_sample_of_cold_rows_of_tiny_logits(n, dtype):
    """Logits and temperatures of about 10^-30 and down to the smallest floats, positive, negative and both."""
    g = gen(n + 3)
    rows = 8
    size = torch.tensor([1e-30, 1e-30, 1e-34, 1e-37, 1e-38, 3e-39, 1e-24, 1e-15], device="cuda").double()[:, None]
    x = (normal(g, rows, n).double() + torch.tensor([0.0, -9.0, 9.0, 0.0, 0.0, 0.0, 3.0, 0.0], device="cuda").double()[:, None]) * size
    x = x.float().to(TD[dtype])
    heat = (size[:, 0] * 0.7).float().clamp(max=9e-21)
    for case in (dict(), dict(k=i32([1, 2, 30, 64, 65, 100, 200, 256])), dict(p=f32([0.5, 0.9, 0.99, 0.3, 0.7, 0.95, 0.8, 0.6])), dict(k=i32([50] * rows), p=f32([0.9] * rows)), dict(m=f32([0.05] * rows))):
        sample_check(x, dtype, t=heat, u=uniform(g, rows), **case)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [513, 2048, 16385, 100000])
def test_sample_of_evenly_spaced_logits(n, dtype):
    """Differences that are whole multiples of a step, so that logits lie on the borders of whatever equal intervals they are sorted into."""
    g = gen(n + 4)
    rows = 10
    steps = torch.tensor([2.0 ** -10, 2.0 ** -7, 2.0 ** -4, 1e-3, 1 / 3, 0.7, 2.0 ** -12, 0.01, 1.0, 8.0], device="cuda")
    order = torch.stack([torch.randperm(n, generator=g, device="cuda") for _ in range(rows)]).float()
    x = (5.0 - order * steps[:, None]).to(TD[dtype])
    ks = [2, 3, 17, 64, 65, 128, 255, 256, 257, 500]
    for case in (dict(k=i32(ks)), dict(k=i32(ks[::-1])), dict(p=f32([0.1, 0.5, 0.75, 0.9, 0.99, 0.999, 0.5, 0.9, 0.3, 0.6])), dict(t=steps * 40, p=f32([0.9] * rows)), dict(t=steps * 3000, p=f32([0.8] * rows)),
                 dict(t=steps * 300, k=i32(ks), p=f32([0.95] * rows))):
        sample_check(x, dtype, u=uniform(g, rows), **case)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,shift", [(1001, 1), (16001, 3), (33333, 5)])
def test_sample_off_a_16_byte_boundary(dtype, n, shift):
    g = gen(shift)
    x = (3 * normal(g, 7, n)).to(TD[dtype])
    k, p, u = i32([0, 5, 60, 700, 0, 9, 0]), f32([0.9, 1, 0.8, 0.95, 1, 0.5, 0.99]), uniform(g, 7)
    sample_check(moved(x, shift), dtype, k=k, p=p, u=u, shift=shift)


def test_sample_in_place_and_probabilities_alone():
    g = gen(4)
    for n in (800, 40000):
        x = 3 * normal(g, 5, n)
        p = f32([0.9] * 5)
        u = uniform(g, 5)
        tokens, out = sample_run(x, "f32", p=p, u=u)
        y = x.clone()
        eb.sample("f32", y, 5, n, None, None, top_p=p, probs=y)
        assert torch.equal(y, out)
        y, other = x.clone(), torch.empty(5, dtype=torch.int32, device="cuda")
        eb.sample("f32", y, 5, n, u, other, top_p=p, probs=y)
        assert torch.equal(y, out) and torch.equal(other, tokens)


def test_sample_draws_what_it_says():
    """20000 draws from one row: each class as often as its probability, within five deviations."""
    g = gen(6)
    rows, n = 20000, 50
    x = normal(g, 1, n).expand(rows, n).contiguous()
    tokens, out = sample_run(x, "f32", k=i32([30] * rows), p=f32([0.9] * rows), u=uniform(g, rows))
    share = torch.bincount(tokens.long(), minlength=n).double() / rows
    q = out[0].double()
    assert bool(((share - q).abs() <= 5 * torch.sqrt(q * (1 - q) / rows)).all())


# ----------------------------------------------------------------------------- together

def test_a_head_in_8_bits_drawn_and_verified():
    """Pooled features quantised, two heads in 8 bits (an early and a later exit), the early one's draws verified against the later one's probabilities."""
    g = gen(10)
    batch, k, c, n = 6, 3, 512, 1000
    feat = normal(g, batch * (k + 1), c).to(torch.bfloat16)
    heads = [quantised((normal(g, n, c) * s * c ** -0.5).to(torch.bfloat16), "bf16") for s in (3.0, 3.2)]
    q, xs = quantised(feat, "bf16")
    probs, drafts = [], None
    for i, (w, ws) in enumerate(heads):
        logits = torch.empty(batch * (k + 1), n, device="cuda")
        eb.int8_linear("f32", q, batch * (k + 1), c, w, ws, n, logits, x_scale=xs)
        tokens, out = sample_run(logits, "f32", t=f32([0.8] * batch * (k + 1)), k=i32([50] * batch * (k + 1)), p=f32([0.95] * batch * (k + 1)), u=uniform(g, batch * (k + 1)))
        probs.append(out.view(batch, k + 1, n))
        drafts = tokens.view(batch, k + 1)[:, :k].contiguous() if i == 0 else drafts
    u, r = uniform(g, batch, k), uniform(g, batch)
    said, accepted = torch.empty(batch, k + 1, dtype=torch.int32, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda")
    eb.verify_drafts(probs[1].contiguous(), probs[0][:, :k].contiguous(), drafts, u, r, batch, k, n, said, accepted)
    for b in range(batch):
        got = int(accepted[b])
        assert all(float(u[b, j]) * float(probs[0][b, j, drafts[b, j]]) < float(probs[1][b, j, drafts[b, j]]) for j in range(got))
        assert said[b, :got].tolist() == drafts[b, :got].tolist() and float(probs[1][b, got, said[b, got]]) > 0
    eb.operators_check()


def test_parked_maps_resumed_in_another_order():
    """Survivors of two batches put away behind one another in a pool, read back as one batch in the order of their resumption, then normed."""
    g = gen(11)
    hw, c = 49, 256
    maps = [normal(g, b, hw, c).to(torch.bfloat16) for b in (3, 5)]
    q = torch.empty(8 * hw, c, dtype=torch.int8, device="cuda")
    scale = torch.empty(8 * hw, device="cuda")
    at = 0
    for m in maps:
        eb.quantize_rows("bf16", m, m.shape[0] * hw, c, q[at:], scale[at:])
        at += m.shape[0] * hw
    order = [6, 1, 3]
    index = torch.cat([torch.arange(i * hw, (i + 1) * hw) for i in order]).int().cuda()
    batch = torch.empty(3, hw, c, dtype=torch.bfloat16, device="cuda")
    eb.dequantize_rows("bf16", q, scale, 8 * hw, c, batch, 3 * hw, index=index)
    want = torch.cat(maps)[order].view(3 * hw, c)
    big = want.double().abs().amax(1, keepdim=True)
    # half a step of about 1/127 of the row's largest, then the rounding of the value
    assert bool(((batch.view(3 * hw, c).double() - want.double()).abs() <= big / 254 * 1.0001 + HALF["bf16"] * want.double().abs() * 1.01 + 2.0 ** -8 * big / 254).all())
    y = torch.empty_like(batch)
    eb.group_norm("bf16", batch, 3, hw, c, 8, None, None, 1e-5, 1, y)
    assert bool(torch.isfinite(y).all())


# ----------------------------------------------------------------------------- streams, graphs, devices

def test_other_streams_and_captured_graphs():
    g = gen(12)
    x, w, ws, bias = linear_case(70, 600, 900, "bf16")
    w8 = padded(w)
    rows, n = 70, 900
    room = [torch.empty(eb.int8_linear_workspace_bytes(rows, 600) + 256, dtype=torch.uint8, device="cuda") for _ in range(2)]
    u = uniform(g, rows)

    def pass_(x, y, tokens, probs, room, stream=None):
        eb.int8_linear("bf16", x, rows, 600, w8, ws, n, y, workspace=room, bias=bias, stream=stream)
        eb.sample("bf16", y, rows, n, u, tokens, top_k=i32_50, top_p=p9, probs=probs, stream=stream)

    i32_50, p9 = i32([50] * rows), f32([0.9] * rows)
    new = lambda: (torch.empty(rows, n, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, n, device="cuda"))  # noqa: E731
    want = new()
    pass_(x, *want, room[0])
    outs = [new(), new()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):                       # two streams at once, a workspace each
        for o, r, s in zip(outs, room, streams):
            pass_(x, *o, r, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(o, want))
    held = x.clone()
    captured = new()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pass_(held, *captured, room[0])
    for seed in (1, 2):
        held.copy_(normal(gen(seed), rows, 600).to(torch.bfloat16))
        graph.replay()
        again = new()
        pass_(held, *again, room[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, again))


def test_the_binding_refuses_what_the_library_cannot_see():
    x, q, s = torch.zeros(4, 20, device="cuda"), torch.zeros(4, 32, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    for bad in (dict(x=x.cpu()), dict(x=x.bfloat16()), dict(x=x.t()), dict(q=q[:, :20]), dict(q=q[:3]), dict(q=q.float()), dict(scale=s[:3]), dict(scale=s.double())):
        args = dict(dict(x=x, q=q, scale=s), **bad)
        with pytest.raises(eb.EEError):
            eb.quantize_rows("f32", args["x"], 4, 20, args["q"], args["scale"])
    with pytest.raises(eb.EEError):
        eb.dequantize_rows("f32", q, s, 4, 20, x, 4, index=torch.zeros(4, dtype=torch.int64, device="cuda"))
    with pytest.raises(eb.EEError):
        eb.int8_linear("f32", q, 4, 20, q, s, 4, torch.empty(4, 4, device="cuda"))         # rows of int8 without their scales
    with pytest.raises(eb.EEError):
        eb.int8_linear("f32", x, 4, 20, q, s, 4, torch.empty(4, 4, device="cuda"))         # no workspace
    with pytest.raises(eb.EEError):
        eb.sample("f32", x, 4, 20, s, torch.empty(4, dtype=torch.int64, device="cuda"))
    with pytest.raises(eb.EEError):
        eb.sample("f16", x, 4, 20, s, torch.empty(4, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,n", [(1, 2048, 1000), (3, 4096, 512), (16, 4096, 4096), (40, 4099, 300)])
def test_int8_linear_whose_exchange_runs_out_of_time(rows, c, n, dtype):
    from tests.test_gpu_operator_contracts import _late

    x, w, ws, bias = linear_case(rows, c, n, dtype)
    w8, y = padded(w), torch.empty(rows, n, dtype=TD[dtype], device="cuda")
    room = torch.empty(eb.int8_linear_workspace_bytes(rows, c) + 256, dtype=torch.uint8, device="cuda")
    _late(lambda: eb.int8_linear(dtype, x, rows, c, w8, ws, n, y, workspace=room, bias=bias), [y])
