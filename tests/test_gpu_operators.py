"""The operators that need no model (group norm, adapted projection, softmax, verification of drafts) against their definitions in 64 bits.

Tolerances are sums of the roundings on the way (u = 2^-24, a rounding to fp32; half a step of bf16 is 2^-8 of the value): they are derived beside
each comparison.  Outputs lie in front of canary bytes.
"""
import numpy as np
import pytest
import torch

from paper_2209_13443_b200 import binding as eb
from paper_2209_13443_b200 import workloads as wl
from tests import util

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def out_like(shape, dtype, shift=0):
    """An output tensor filled with a pattern, `shift` elements off its allocation's start, and what must not change around it."""
    n = int(np.prod(shape))
    raw = torch.full((shift + n + 64,), 77.0, dtype=dtype, device="cuda") if dtype.is_floating_point else torch.full((shift + n + 64,), 77, dtype=dtype, device="cuda")
    return raw[shift:shift + n].view(shape), raw


def untouched(raw, shift, n):
    return bool((raw[:shift] == 77).all()) and bool((raw[shift + n:] == 77).all())


def moved(t, shift):
    """The same values, `shift` elements behind a 256-byte boundary."""
    raw = torch.empty(shift + t.numel(), dtype=t.dtype, device="cuda")
    raw[shift:].copy_(t.reshape(-1))
    return raw[shift:].view(t.shape)


# ----------------------------------------------------------------------------- group norm

def norm_exact(x, gamma, beta, groups, eps, act, residual=None):
    b, hw, c = x.shape
    g = x.double().view(b, hw, groups, c // groups)
    var, mean = torch.var_mean(g, (1, 3), correction=0, keepdim=True)
    z = ((g - mean) / torch.sqrt(var + eps)).reshape(b, hw, c)
    t = z * (1.0 if gamma is None else gamma.double()) + (0.0 if beta is None else beta.double())
    if residual is not None:
        t = t + residual.double()
    y = {0: t, 1: t.clamp(min=0), 2: t.clamp(0, 6), 3: t * torch.sigmoid(t)}[act]
    return y, t, z, mean, var


def norm_check(y, x, gamma, beta, groups, eps, act, dtype, residual=None):
    """The mean of n values added by threads (chains of up to m, then a tree) is off by (m + 24) u of the mean magnitude, the sum of squares by that share
    of itself, so a normalised value by (m + 24) u (|x| / deviation + |z|); the affine step, the activation and a residual add a few u of their operands; SiLU's
    exponential is off by 2 + 1.2 |t| units, weighed by a value of at most 0.28 (|t| exp(-t) / (1 + exp(-t))^2 times ...): 4 u + 2 u |t|."""
    ref, t, z, mean, var = norm_exact(x, gamma, beta, groups, eps, act, residual)
    b, hw, c = x.shape
    m = max(32.0, hw / 16.0 if c // groups >= 4 else hw / 4.0)
    big = x.double().abs().view(b, hw, groups, c // groups).amax((1, 3), keepdim=True)
    lost = ((m + 24) * U * (big / torch.sqrt(var + eps) + 2 * z.abs().view(b, hw, groups, c // groups))).reshape(b, hw, c)
    if gamma is not None:
        lost = lost * gamma.double().abs()
    tol = lost * 1.1 + 8 * U * (t.abs() + 1) * (2 if act == 3 else 1) + HALF[dtype] * (ref.abs() + lost)
    if residual is not None:
        tol = tol + 2 * U * residual.double().abs()
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), f"off by {float((err / tol).max()):.3g} tolerances"


NORMS = [  # batch, hw, c, groups
    (1, 1, 1, 1), (1, 1, 8, 8), (2, 1, 64, 4), (3, 2, 40, 5), (1, 49, 2048, 32), (2, 957, 96, 32), (3, 100, 30, 30), (2, 63, 37, 1), (2, 9, 1001, 1), (1, 5, 6006, 6),
    (1, 10, 4096, 1), (2, 17, 600, 2), (2, 3136, 64, 8), (1, 12544, 96, 8), (1, 60001, 64, 4), (1, 20000, 3, 1), (1, 65, 512, 512), (5, 33, 24, 2), (1, 2, 16384, 4), (64, 4, 48, 6),
    (1, 100003, 24, 8), (1, 30000, 520, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", NORMS, ids=str)
def test_group_norm(shape, dtype):
    b, hw, c, groups = shape
    g = gen(b + hw + c)
    x = (normal(g, b, hw, c) * (0.5 + normal(g, c).abs()) + 1.5 * normal(g, c)).to(TD[dtype])
    gamma, beta = 1 + 0.2 * normal(g, c), 0.1 * normal(g, c)
    act = (hw + c) % 4
    y, raw = out_like(x.shape, TD[dtype])
    eb.group_norm(dtype, x, b, hw, c, groups, gamma, beta, 1e-5, act, y)
    norm_check(y, x, gamma, beta, groups, 1e-5, act, dtype)
    assert untouched(raw, 0, x.numel())
    # a sample's bits do not depend on the batch, nor on the address
    alone, raw = out_like(x[:1].shape, TD[dtype])
    eb.group_norm(dtype, x[b - 1:].contiguous(), 1, hw, c, groups, gamma, beta, 1e-5, act, alone)
    assert torch.equal(alone[0], y[b - 1])


@pytest.mark.parametrize("act", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_group_norm_with_a_residual_and_in_place(dtype, act):
    b, hw, c, groups = 3, 196, 128, 8
    g = gen(act)
    x, res = (3 * normal(g, b, hw, c)).to(TD[dtype]), normal(g, b, hw, c).to(TD[dtype])
    gamma, beta = 1 + normal(g, c), normal(g, c)
    y, raw = out_like(x.shape, TD[dtype])
    eb.group_norm(dtype, x, b, hw, c, groups, gamma, beta, 1e-3, act, y, residual=res)
    norm_check(y, x, gamma, beta, groups, 1e-3, act, dtype, residual=res)
    assert untouched(raw, 0, x.numel())
    for into in ("x", "residual"):
        xi, ri = x.clone(), res.clone()
        eb.group_norm(dtype, xi, b, hw, c, groups, gamma, beta, 1e-3, act, xi if into == "x" else ri, residual=ri)
        assert torch.equal(xi if into == "x" else ri, y)
    eb.group_norm(dtype, x, b, hw, c, groups, None, None, 1e-3, act, y)
    norm_check(y, x, None, None, groups, 1e-3, act, dtype)


@pytest.mark.parametrize("dtype,shifts", [("f32", (1, 0, 0)), ("f32", (0, 3, 2)), ("bf16", (1, 1, 1)), ("bf16", (0, 0, 5)), ("bf16", (4, 0, 0))])
def test_group_norm_off_a_16_byte_boundary(dtype, shifts):
    b, hw, c, groups = 2, 50, 64, 4
    g = gen(5)
    x, res = normal(g, b, hw, c).to(TD[dtype]), normal(g, b, hw, c).to(TD[dtype])
    y, raw = out_like(x.shape, TD[dtype], shifts[2])
    eb.group_norm(dtype, moved(x, shifts[0]), b, hw, c, groups, None, None, 1e-5, 1, y, residual=moved(res, shifts[1]))
    norm_check(y, x, None, None, groups, 1e-5, 1, dtype, residual=res)
    assert untouched(raw, shifts[2], x.numel())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [100.0, -3000.0])
def test_group_norm_of_a_large_mean(dtype, offset):
    """Statistics about the mean: with sums of squares alone a mean of 3000 deviations leaves nothing of the variance in fp32."""
    g = gen(9)
    x = (normal(g, 2, 3000, 32) + offset).to(TD[dtype])
    y, _ = out_like(x.shape, TD[dtype])
    eb.group_norm(dtype, x, 2, 3000, 32, 2, None, None, 1e-5, 0, y)
    norm_check(y, x, None, None, 2, 1e-5, 0, dtype)


def test_group_norm_of_constant_and_non_finite_groups():
    x = torch.full((2, 40, 16), 2.0, device="cuda")
    x[1, 3, 9] = float("inf")
    x[1, 7, 1] = float("nan")
    y, _ = out_like(x.shape, torch.float32)
    eb.group_norm("f32", x, 2, 40, 16, 4, None, None, 1e-5, 0, y)
    assert torch.equal(y[0], torch.zeros_like(y[0]))                       # no deviation: (x - mean) = 0
    v = y[1].view(40, 4, 4)
    assert bool(v[:, [0, 2]].isnan().all()) and bool((v[:, [1, 3]] == 0).all())    # only the groups that hold them
    eb.group_norm("f32", x[:1].contiguous(), 1, 40, 16, 4, None, None, 0.0, 0, y)
    assert bool(y[0].isnan().all())                                        # 0 / 0, as the formula has it


# ----------------------------------------------------------------------------- adapted projection

def linear_operands(seed, rows, c, n, rank, adapters, dtype, order="mixed"):
    g = gen(seed)
    td = TD[dtype]
    x, w = normal(g, rows, c).to(td), (normal(g, n, c) * c ** -0.5).to(td)
    a, b = (normal(g, adapters, rank, c) * c ** -0.5).to(td), normal(g, adapters, n, rank).to(td)
    which = torch.randint(-1, adapters, (rows,), generator=g, device="cuda")
    if order == "runs":
        which = torch.sort(which)[0]
    elif order == "none":
        which = torch.full_like(which, -1)
    elif order == "one":
        which = torch.full_like(which, adapters - 1)
    elif order == "strange":
        which = torch.where(which < 0, torch.full_like(which, adapters + 3), which)
        which[::3] = -(2 ** 31)
    return x, w, normal(g, n), a, b, 0.5 + torch.rand(adapters, generator=g, device="cuda"), which.int()


def linear_check(y, x, w, bias, a, b, scale, which, dtype):
    """Products of bf16 values are exact in fp32; a sum of c of them, added 16 at a time with what the tensor core drops, is off by at most (c / 16 + 20) 2 u of the sum of
    magnitudes S.  The adapter's share: h off by that of |A||x|, its two bf16 parts by 2^-17, the rest as above.  fp32: sums in fp64; h, its scaled
    value and the share itself are rounded to fp32."""
    x, w, a, b = x.double(), w.double(), a.double(), b.double()
    rows, c = x.shape
    y64, mag = x @ w.t(), x.abs() @ w.abs().t()
    share = torch.zeros_like(mag)
    for i in range(a.shape[0]):
        r = (which == i).nonzero()[:, 0]
        s = 1.0 if scale is None else float(scale[i])
        y64[r] += s * ((x[r] @ a[i].t()) @ b[i].t())
        share[r] += s * ((x[r].abs() @ a[i].abs().t()) @ b[i].abs().t())
    if bias is not None:
        y64, mag = y64 + bias.double(), mag + bias.double().abs()
    if dtype == "bf16":
        k = (c / 16 + 20) * 2 * U
        lost = k * (mag + 2 * share) + 2.0 ** -17 * share
    else:
        lost = 4 * U * share + U * y64.abs()
    tol = lost + HALF[dtype] * (y64.abs() + lost)
    err = (y.double() - y64).abs()
    assert bool((err <= tol).all()), f"off by {float((err / tol).max()):.3g} tolerances"


def linear_run(dtype, ops, with_bias=True, with_scale=True, shifts=(0, 0, 0, 0, 0)):
    x, w, bias, a, b, scale, which = ops
    (rows, c), n, (m, rank, _) = x.shape, w.shape[0], a.shape
    x, w, a, b = (moved(t, s) if s else t for t, s in zip((x, w, a, b), shifts))
    y, raw = out_like((rows, n), TD[dtype], shifts[4])
    need = eb.adapted_linear_workspace_bytes(rows, rank)
    ws, guard = util.guarded((need,), torch.uint8)
    ws.fill_(0xff)                                         # NaN wherever a sum was not written
    eb.adapted_linear(dtype, x, rows, c, w, n, a, b, rank, m, which, y, ws, bias=bias if with_bias else None, scale=scale if with_scale else None)
    assert untouched(raw, shifts[4], rows * n) and bool((guard == util.CANARY).all())
    linear_check(y, ops[0], ops[1], bias if with_bias else None, ops[3], ops[4], scale if with_scale else None, which, dtype)
    eb.operators_check()
    return y


LINEARS = [  # rows, c, n, rank, adapters
    (1, 8, 1, 1, 1), (1, 2048, 1000, 8, 16), (2, 64, 40, 3, 2), (5, 200, 129, 16, 3), (16, 512, 256, 64, 16), (17, 320, 130, 5, 40), (32, 1024, 384, 128, 7), (33, 72, 512, 9, 4), (64, 4096, 512, 16, 32),
    (96, 128, 200, 8, 3), (97, 136, 300, 24, 97), (128, 256, 128, 128, 128), (129, 264, 257, 33, 5), (200, 648, 1000, 64, 9), (300, 64, 64, 8, 300), (513, 1032, 640, 16, 6), (1100, 512, 4096, 4, 3)]


@pytest.mark.parametrize("order", ["mixed", "runs"])
@pytest.mark.parametrize("shape", LINEARS, ids=str)
def test_adapted_linear_bf16(shape, order):
    linear_run("bf16", linear_operands(sum(shape), *shape, "bf16", order))


@pytest.mark.parametrize("shape", [(1, 2048, 100, 8, 4), (3, 7, 5, 3, 2), (37, 2048, 1000, 5, 7), (70, 130, 33, 128, 70), (256, 512, 300, 16, 9), (40, 100, 200, 64, 3)], ids=str)
def test_adapted_linear_f32(shape):
    linear_run("f32", linear_operands(sum(shape), *shape, "f32"))


@pytest.mark.parametrize("shape", [(1, 7, 9, 3, 2), (3, 65, 200, 17, 5), (20, 2, 130, 1, 3), (40, 130, 100, 12, 9), (70, 1001, 77, 8, 4), (150, 514, 300, 40, 33), (300, 999, 129, 7, 11)], ids=str)
def test_adapted_linear_of_channels_that_are_not_whole_vectors(shape):
    linear_run("bf16", linear_operands(sum(shape), *shape, "bf16"))


@pytest.mark.parametrize("dtype,rows,shifts", [("bf16", 9, (1, 0, 0, 0, 0)), ("bf16", 150, (0, 2, 0, 0, 1)), ("bf16", 150, (0, 0, 1, 4, 0)), ("bf16", 40, (0, 0, 0, 1, 3)), ("f32", 20, (1, 0, 2, 3, 1)),
                                               ("f32", 50, (0, 1, 1, 0, 0))])
def test_adapted_linear_off_a_16_byte_boundary(dtype, rows, shifts):
    linear_run(dtype, linear_operands(3, rows, 256, 200, 16, 6, dtype), shifts=shifts)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [12, 140])
@pytest.mark.parametrize("order", ["none", "one", "strange"])
def test_adapted_linear_rows_without_or_with_one_adapter(dtype, rows, order):
    ops = linear_operands(rows, rows, 320, 256, 16, 5, dtype, order)
    y = linear_run(dtype, ops, with_bias=False, with_scale=False)
    if order == "none":       # the plain projection, bit for bit
        x, w = ops[0], ops[1]
        plain, _ = out_like(y.shape, TD[dtype])
        eb.adapted_linear(dtype, x, rows, 320, w, 256, None, None, 0, 0, None, plain, None)
        assert torch.equal(plain, y)


def test_adapted_linear_keeps_other_rows_out_of_a_row():
    """Adapters of NaN: rows that do not name them stay what they are."""
    for rows in (20, 200):
        x, w, bias, a, b, scale, which = linear_operands(8, rows, 512, 256, 8, 4, "bf16")
        y = linear_run("bf16", (x, w, bias, a, b, scale, which))
        ops_a, a, b = a, a.clone(), b.clone()
        a[2] = float("nan")
        b[1] = float("inf")
        b[1, 5:] = -float("inf")
        bad, _ = out_like(y.shape, torch.bfloat16)
        ws = torch.empty(eb.adapted_linear_workspace_bytes(rows, 8), dtype=torch.uint8, device="cuda")
        eb.adapted_linear("bf16", x, rows, 512, w, 256, a, b, 8, 4, which, bad, ws, bias=bias, scale=scale)
        clean = (which != 1) & (which != 2)
        same = bad[clean] == y[clean]
        assert bool(bad[which == 2].isnan().all())
        one = (which == 1).nonzero()[:, 0]                 # infinities of both signs in one sum are NaN; a row of one sign is that
        h = x[one].double() @ ops_a[1].double().t()
        same_sign = (h > 0).all(1) | (h < 0).all(1)
        assert bool((~bad[one].isfinite()).all()) and torch.equal(bad[one][:, 0].isinf(), same_sign) and torch.equal(bad[one][:, 9].isinf(), same_sign)
        assert bool(same.all()), "a row took something of an adapter that is not its own"


# ----------------------------------------------------------------------------- softmax

def softmax_exact(x, heat):
    z = x.double()
    t = torch.ones(x.shape[0], dtype=torch.float64, device="cuda") if heat is None else heat.double()
    out = torch.zeros_like(z)
    for i in range(x.shape[0]):
        row = z[i]
        if bool(row.isnan().any()) or bool((row == float("inf")).any()):
            out[i] = float("nan")
        elif bool((row == float("-inf")).all()):
            pass
        elif not float(t[i]) > 0:
            out[i, int((row == row.max()).nonzero()[0])] = 1.0
        else:
            e = torch.exp((row - row.max()) / t[i])
            out[i] = e / e.sum()
    return out


def softmax_check(y, x, heat):
    """The exponent (l - max) / t is off by 4 u of itself (difference, constant, quotient, product), the power by 2 units of 2 u, twice where a row is cut; the sum's chain is n / 512 and
    its tree 16 long, the quotient and its product 2 u.  What underflows is off by the smallest normal number."""
    ref = softmax_exact(x, heat)
    n = x.shape[1]
    fin = ref.isfinite()
    assert torch.equal(fin, y.isfinite())
    d = torch.log(ref.clamp(min=1e-300)).abs()           # |l - max| / t + log(sum) >= |l - max| / t
    tol = ref * U * (5 * d + 20 + n / 512 + 32) + 2.0 ** -126
    err = torch.where(fin, (y.double() - ref).abs(), torch.zeros_like(ref))
    assert bool((err <= tol)[fin].all()), f"off by {float((err / tol)[fin].max()):.3g} tolerances"
    assert bool((y[ref == 0] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 1), (5, 2), (3, 31), (9, 128), (7, 129), (64, 1000), (3, 1024), (3, 1025), (4, 4099), (2, 16385), (3, 32769), (2, 50001), (3, 128001), (1, 262145), (2, 409600), (1, 614399)])
def test_softmax(rows, n, dtype):
    g = gen(n)
    x = (3 * normal(g, rows, n)).to(TD[dtype])
    y, raw = out_like((rows, n), torch.float32)
    eb.softmax(dtype, x, rows, n, y)
    softmax_check(y, x, None)
    assert untouched(raw, 0, rows * n)
    heat = 0.3 + torch.rand(rows, generator=g, device="cuda")
    heat[0] = 0.0                                          # the largest logit alone
    x[rows - 1, : n // 2] = float("-inf")
    eb.softmax(dtype, x, rows, n, y, temperature=heat)
    softmax_check(y, x, heat)
    again, raw = out_like((1, n), torch.float32, 1)        # another place in memory, another batch: the same bits
    eb.softmax(dtype, moved(x[rows - 1], 3).view(1, n), 1, n, again, temperature=heat[rows - 1:].contiguous())
    assert torch.equal(again[0], y[rows - 1]) and untouched(raw, 1, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [40, 900, 5000, 70001])
def test_softmax_of_masked_and_non_finite_rows(n, dtype):
    g = gen(1)
    x = normal(g, 10, n).to(TD[dtype])
    low, inf, nan = torch.finfo(TD[dtype]).min, float("inf"), float("nan")
    x[0] = -inf                                            # nothing left: all 0
    x[1] = low                                             # the type's lowest value is a number: uniform
    x[2, 5:] = -inf
    x[3, 7:] = low
    x[4, 3] = nan
    x[5, n - 1] = inf
    x[6, 9], x[6, n - 2] = 50.0, 50.0                      # a tie
    x[7] = nan
    heat = torch.ones(10, device="cuda")
    y, raw = out_like((10, n), torch.float32)
    for t in (None, heat, heat * 1e-30, heat * 1e-45, heat * 1e30, heat * inf, -heat, heat * 0, heat * nan):
        eb.softmax(dtype, x, 10, n, y, temperature=t)
        if t is None or float(t[0]) == 1.0:
            softmax_check(y, x, t)
        elif not float(t[0]) > 0 or float(t[0]) < 1e-20:
            exact = softmax_exact(x, -heat)
            if float(t[0]) > 0:                            # so cold that only ties share
                exact[1], exact[6] = 1.0 / n, (x[6] == x[6].max()).double() / 2
            assert torch.equal(y.isnan(), exact.isnan()) and torch.allclose(y.double().nan_to_num(), exact.nan_to_num(), rtol=1e-6, atol=0)
        else:                                              # so hot that all that are left share (the lowest value may still be infinitely far)
            assert bool(y[4].isnan().all() and y[5].isnan().all() and y[7].isnan().all()) and bool((y[0] == 0).all())
            assert torch.allclose(y[2, :5], torch.full((5,), 0.2, device="cuda"), rtol=1e-6) and bool((y[2, 5:] == 0).all())
    assert untouched(raw, 0, 10 * n)


def test_softmax_in_place():
    for n in (300, 20000):
        x = normal(gen(n), 4, n)
        y, _ = out_like((4, n), torch.float32)
        eb.softmax("f32", x, 4, n, y)
        eb.softmax("f32", x, 4, n, x)
        assert torch.equal(x, y)


# ----------------------------------------------------------------------------- verification

def verify_exact(p, q, drafts, u, r, count, tokens, accepted):
    """The procedure as ee.h tells it, in fp64; rows of a negative count keep what tokens and accepted hold."""
    b, k1, n = p.shape
    k = k1 - 1
    p = p.double().cpu().numpy()
    q = None if q is None else q.double().cpu().numpy()
    drafts, u, r = drafts.cpu().numpy(), u.double().cpu().numpy(), r.double().cpu().numpy()
    tokens, accepted = tokens.cpu().numpy().copy(), accepted.cpu().numpy().copy()
    for i in range(b):
        have = k if count is None else min(int(count[i]), k)
        if have < 0:
            continue
        j = 0
        while j < have:
            t = int(drafts[i, j])
            if not (0 <= t < n) or not u[i, j] * (1.0 if q is None else q[i, j, t]) < p[i, j, t]:
                break
            j += 1

        def weights(minus):
            with np.errstate(invalid="ignore"):
                w = p[i, j] - minus
            w[~((w > 0) & (w < np.inf))] = 0.0
            return w
        w = weights(0.0)
        if j < have:
            if q is None:
                left = w.copy()
                if 0 <= drafts[i, j] < n:
                    left[drafts[i, j]] = 0.0
            else:
                left = weights(q[i, j])
            if left.sum() > 0:
                w = left
        cum = np.cumsum(w)
        token = -1
        if cum[-1] > 0:
            goal = r[i] * cum[-1] if r[i] > 0 else 0.0          # NaN counts as 0
            over = (cum > goal) & (w > 0)
            token = int(over.argmax()) if over.any() else int(np.flatnonzero(w > 0)[-1])
        tokens[i] = -1
        tokens[i, :j] = drafts[i, :j]
        tokens[i, j] = token
        accepted[i] = j
    return tokens, accepted


def verify_case(p, q, drafts, u, r, count=None, stream=None):
    b, k1, n = p.shape
    tokens, raw_t = out_like((b, k1), torch.int32)
    accepted, raw_a = out_like((b,), torch.int32)
    want_t, want_a = verify_exact(p, q, drafts, u, r, None if count is None else count.tolist(), tokens, accepted)
    eb.verify_drafts(p, q, drafts, u, r, b, k1 - 1, n, tokens, accepted, n_draft=count, stream=stream)
    assert np.array_equal(accepted.cpu().numpy(), want_a)
    assert np.array_equal(tokens.cpu().numpy(), want_t)
    assert untouched(raw_t, 0, b * k1) and untouched(raw_a, 0, b)
    return tokens, accepted


def drafts_of(seed, b, k, n, spread=0.7):
    g = gen(seed)
    base = 2.5 * normal(g, b, k + 1, n)
    p, q = torch.softmax(base, -1), torch.softmax(base[:, :k] + spread * normal(g, b, k, n), -1)
    d = torch.multinomial(q.reshape(b * k, n), 1, generator=g).view(b, k).int() if k else torch.zeros((b, 0), dtype=torch.int32, device="cuda")
    return p, q, d, torch.rand((b, k), generator=g, device="cuda"), torch.rand(b, generator=g, device="cuda")


@pytest.mark.parametrize("dense", [True, False])
@pytest.mark.parametrize("b,k,n", [(1, 1, 1), (3, 2, 2), (1, 0, 1000), (1, 1, 1000), (70, 4, 33), (5, 40, 100), (9, 3, 8192), (9, 3, 8193), (4, 2, 20001), (3, 5, 65537), (4, 5, 128001), (1, 1, 2300001)])
def test_verify_drafts(b, k, n, dense):
    p, q, d, u, r = drafts_of(b + k + n, b, k, n)
    verify_case(p, q if dense else None, d, u, r)
    g = gen(n)
    count = torch.randint(-1, k + 3, (b,), generator=g, device="cuda").int()
    verify_case(p, q if dense else None, d, u, r, count)
    verify_case(p, q if dense else None, d, u * 0, r * 0)              # r = 0: the first that weighs anything
    verify_case(p, q if dense else None, d, u * 0 + 1 - 2.0 ** -24, r * 0 + 1 - 2.0 ** -24)


@pytest.mark.parametrize("n", [50, 3000, 40001])
def test_verify_drafts_of_odd_rows(n):
    inf, nan = float("inf"), float("nan")
    p, q, d, u, r = drafts_of(n, 12, 2, n)
    d[0, 0], d[1, 1], d[2, 0] = -5, n, 2 ** 31 - 1                      # no classes
    p[3], q[4, 0] = 0.0, 2.0                                            # nothing to draw from; q above p everywhere
    p[5, :, ::2], q[6, :, 1::3] = nan, inf
    p[7, :, n // 2] = inf
    p[8] = 0.0
    p[8, :, n - 1] = 1e-30                                              # one that weighs anything, the last one
    q[9] = p[9, :2]                                                     # equal: everything is accepted
    p[10] = -1.0
    p[11, 0], d[11, 0], u[11, 0] = 0.0, 0, 0.0                          # u = 0 does not accept what is impossible
    verify_case(p, q, d, u, r)
    verify_case(p, None, d, u, r)
    verify_case(p, q, d, u * nan, r * nan)                              # no number is below another: all rejected, the first that weighs anything
    verify_case(p, q, d, u, r * 0 + 2.0)                                # beyond the total: the last one that weighs anything


def test_verified_answers_are_distributed_as_the_target():
    """What verification gives out for the first position of many sequences follows p, whoever drafted: mean counts within six deviations."""
    b, n = 20000, 7
    g = gen(0)
    row_p, row_q = torch.softmax(normal(g, n), 0), torch.softmax(normal(g, n), 0)
    p, q = row_p.expand(b, 2, n).contiguous(), row_q.expand(b, 1, n).contiguous()
    d = torch.multinomial(q.view(b, n), 1, generator=g).int()
    u, r = torch.rand((b, 1), generator=g, device="cuda"), torch.rand(b, generator=g, device="cuda")
    tokens = torch.empty((b, 2), dtype=torch.int32, device="cuda")
    accepted = torch.empty(b, dtype=torch.int32, device="cuda")
    eb.verify_drafts(p, q, d, u, r, b, 1, n, tokens, accepted)
    share = torch.bincount(tokens[:, 0].long(), minlength=n).double() / b
    assert bool(((share - row_p.double()).abs() < 6 * torch.sqrt(row_p.double() / b)).all())


# ----------------------------------------------------------------------------- how they are called

def test_a_branch_of_all_of_them():
    """An exit branch as many requests share it: the map is normalised, pooled, projected through every request's own head by an early and a final
    exit, and the early answers are verified against the final ones; in a captured graph, replayed on other inputs, and eagerly on another stream."""
    b, hw, c, n, rank, m = 24, 49, 256, 1000, 8, 5
    g = gen(4)
    x = torch.empty((b, hw, c), dtype=torch.bfloat16, device="cuda")
    gamma, beta = 1 + 0.1 * normal(g, c), 0.1 * normal(g, c)
    w, a, bb = [(normal(g, n, c) * 0.2).bfloat16() for _ in range(2)], (normal(g, m, rank, c) * c ** -0.5).bfloat16(), normal(g, m, n, rank).bfloat16()
    which = torch.randint(-1, m, (b,), generator=g, device="cuda").int()
    u, r = torch.rand((b, 1), generator=g, device="cuda"), torch.rand(b, generator=g, device="cuda")
    draft = torch.empty((b, 1), dtype=torch.int32, device="cuda")

    def buffers():
        return dict(y=torch.empty_like(x), pooled=torch.empty((b, c), dtype=torch.bfloat16, device="cuda"), z=[torch.empty((b, n), dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                    q=torch.empty((b, 1, n), device="cuda"), late=torch.empty((b, n), device="cuda"), p=torch.empty((b, 2, n), device="cuda"),
                    ws=torch.empty(eb.adapted_linear_workspace_bytes(b, rank), dtype=torch.uint8, device="cuda"),
                    tokens=torch.empty((b, 2), dtype=torch.int32, device="cuda"), accepted=torch.empty(b, dtype=torch.int32, device="cuda"))

    def branch(o, stream):
        eb.group_norm("bf16", x, b, hw, c, 32, gamma, beta, 1e-5, eb_silu, o["y"], stream=stream)
        o["pooled"].copy_(o["y"].float().mean(1))
        for e in range(2):
            eb.adapted_linear("bf16", o["pooled"], b, c, w[e], n, a, bb, rank, m, which, o["z"][e], o["ws"], stream=stream)
        eb.softmax("bf16", o["z"][0], b, n, o["q"], stream=stream)
        eb.softmax("bf16", o["z"][1], b, n, o["late"], stream=stream)
        draft.copy_(o["q"].argmax(2))
        o["p"].copy_(o["late"][:, None].expand(b, 2, n))
        eb.verify_drafts(o["p"], o["q"], draft, u, r, b, 1, n, o["tokens"], o["accepted"], stream=stream)

    eb_silu = wl.ACT_SILU
    one, two = buffers(), buffers()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    x.copy_(normal(g, b, hw, c))
    torch.cuda.synchronize()
    with torch.cuda.stream(s1):
        branch(one, s1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s1):
        branch(one, s1)
    for seed in range(3):
        x.copy_(normal(gen(seed), b, hw, c))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(s2):
            branch(two, s2)
        torch.cuda.synchronize()
        for k in ("y", "pooled", "q", "p", "tokens", "accepted"):
            assert torch.equal(one[k], two[k]), k
        norm_check(two["y"], x, gamma, beta, 32, 1e-5, 3, "bf16")
        for e in range(2):
            linear_check(two["z"][e], two["pooled"], w[e], None, a, bb, None, which, "bf16")
        softmax_check(two["late"], two["z"][1], None)
        want_t, want_a = verify_exact(two["p"], two["q"], draft, u, r, None, two["tokens"], two["accepted"])
        assert np.array_equal(two["tokens"].cpu().numpy(), want_t) and np.array_equal(two["accepted"].cpu().numpy(), want_a)
    eb.operators_check()


def test_two_calls_at_once_with_a_workspace_each():
    ops = [linear_operands(i, 64, 2048, 1024, 16, 8, "bf16") for i in range(2)]
    want = [linear_run("bf16", o) for o in ops]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(y) for y in want]
    wss = [torch.empty(eb.adapted_linear_workspace_bytes(64, 16), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for (x, w, bias, a, b, scale, which), y, ws, st in zip(ops, outs, wss, streams):
            eb.adapted_linear("bf16", x, 64, 2048, w, 1024, a, b, 16, 8, which, y, ws, bias=bias, scale=scale, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("what", ["type", "place", "size", "strides", "dtype", "workspace"])
def test_the_binding_refuses_operands_that_do_not_fit(what):
    x, y = torch.zeros((2, 9, 16), device="cuda"), torch.zeros((2, 9, 16), device="cuda")
    gamma, dtype, n = None, "f32", 9
    if what == "type":
        x = x.double()
    elif what == "place":
        gamma = torch.ones(16)
    elif what == "size":
        n = 10
    elif what == "strides":
        y = y.transpose(1, 2)
    elif what == "dtype":
        dtype = "f16"
    if what == "workspace":
        ops = linear_operands(0, 5, 64, 32, 8, 2, "bf16")
        with pytest.raises(eb.EEError):
            eb.adapted_linear("bf16", ops[0], 5, 64, ops[1], 32, ops[3], ops[4], 8, 2, ops[6], torch.empty((5, 32), dtype=torch.bfloat16, device="cuda"),
                              torch.empty(eb.adapted_linear_workspace_bytes(5, 8) - 1, dtype=torch.uint8, device="cuda"))
        return
    with pytest.raises(eb.EEError):
        eb.group_norm(dtype, x, 2, n, 16, 4, gamma, None, 1e-5, 0, y)


# ----------------------------------------------------------------------------- group norm as a layer of a stage

def norm_model(dtype, residual_at_norm):
    """Two stages of convolutions normalised by group norm: a stem, and a block whose shortcut is added by its last norm."""
    rng = np.random.default_rng(3)

    def weights(*shape):
        k = int(np.prod(shape[1:]))
        v = (rng.standard_normal(shape) * (2.0 / k) ** 0.5).astype(np.float32)
        return wl.to_bf16_grid(v) if dtype == "bf16" else v

    def vec(n, mean, dev):
        return (mean + dev * rng.standard_normal(n)).astype(np.float32)

    def conv(cin, cout, k, stride=1, **kw):
        return wl.Layer(wl.OP_CONV, cin, cout, k, k, stride, k // 2, wl.ACT_NONE, weight=weights(cout, k, k, cin), scale=None, bias=vec(cout, 0, 0.1), **kw)

    def norm(c, groups, act, **kw):
        return wl.Layer(wl.OP_GROUPNORM, c, c, act=act, scale=vec(c, 1, 0.2), bias=vec(c, 0, 0.1), norm_groups=groups, norm_eps=1e-5, **kw)

    one = [conv(3, 32, 3, 2), norm(32, 8, wl.ACT_SILU)]
    two = [conv(32, 64, 1, 2), norm(64, 16, wl.ACT_NONE), conv(32, 64, 3, 2, input_from=wl.FROM_STAGE_INPUT), norm(64, 16, wl.ACT_RELU),
           conv(64, 64, 3), norm(64, 4, wl.ACT_RELU, residual_from=1 if residual_at_norm else wl.NO_RESIDUAL)]
    stages = [wl.Stage(one, 10, weights(10, 32), vec(10, 0, 0.1), 0.2, False), wl.Stage(two, 10, weights(10, 64), vec(10, 0, 0.1), 0.0, True)]
    return wl.Model(f"norm_{dtype}", dtype, 24, 24, 3, stages, 6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [True, False])
def test_group_norm_as_a_layer(dtype, residual):
    spec = norm_model(dtype, residual)
    m = eb.EEModel(spec)
    bufs = [eb.StageBuffers(m, s) for s in range(2)]
    ws = m.workspace()
    x0 = eb.to_device(dtype, wl.make_input(spec, 6, seed=1))
    singles = []
    for batch in (6, 1):
        feat, n = x0[:batch].contiguous(), batch
        ids = torch.arange(batch, dtype=torch.int32, device="cuda")
        for s in range(2):
            # the stage layer by layer: every norm is the operator itself on what the layer before it left, every convolution the library's own
            outs = []
            for i, l in enumerate(spec.stages[s].layers):
                src = feat[:n].contiguous() if i == 0 or l.input_from == wl.FROM_STAGE_INPUT else outs[i - 1]
                oh, ow = wl.out_hw(src.shape[1], src.shape[2], l)
                y = torch.empty((n, oh, ow, l.cout), dtype=TD[dtype], device="cuda")
                res = outs[l.residual_from] if l.residual_from >= 0 else None
                m.layer_run(s, i, src, res, n, y, ws)
                if l.op == wl.OP_GROUPNORM:
                    gm, bt = torch.from_numpy(l.scale).cuda(), torch.from_numpy(l.bias).cuda()
                    same = torch.empty_like(y)
                    eb.group_norm(dtype, src, n, oh * ow, l.cout, l.norm_groups, gm, bt, l.norm_eps, l.act, same, residual=res)
                    assert torch.equal(same, y)
                    norm_check(y.view(n, oh * ow, -1), src.view(n, oh * ow, -1), gm, bt, l.norm_groups, l.norm_eps, l.act, dtype, None if res is None else res.view(n, oh * ow, -1))
                outs.append(y)
            plan = m.plan(s, n)
            assert [p["kernel"] for p in plan if spec.stages[s].layers[plan.index(p)].op == wl.OP_GROUPNORM] == ["group_norm"] * sum(l.op == wl.OP_GROUPNORM for l in spec.stages[s].layers)
            m.stage_run(s, feat, n, bufs[s], ws, ids)
            torch.cuda.synchronize()
            m.check()
            left = int(bufs[s].n_surv_dev[0])
            stay = bufs[s].survivor_idx[:left].long()
            if s == 0:
                assert torch.equal(bufs[s].features_out[:left], outs[-1][stay])
                # every sample goes on, so that the second stage sees them all
                feat = outs[-1]
                if batch == 6:
                    singles = [outs[-1][0].clone()]
                else:
                    assert torch.equal(outs[-1][0], singles[0])
            else:
                z = outs[-1].double().mean((1, 2)) @ torch.from_numpy(spec.stages[s].fc_weight).double().cuda().t() + torch.from_numpy(spec.stages[s].fc_bias).double().cuda()
                assert float((bufs[s].logits[:n].double() - z).abs().max()) < (1e-5 if dtype == "f32" else 1e-2) * float(z.abs().max())
    m.close()


@pytest.mark.parametrize("changed", [dict(norm_groups=0), dict(norm_groups=5), dict(norm_groups=64), dict(norm_eps=-1.0), dict(norm_eps=float("nan")), dict(kh=3), dict(kw=3), dict(stride=2), dict(pad=1, kh=3, kw=3),
                                     dict(act=4), dict(cout=64)])
def test_group_norm_layers_that_are_refused(changed):
    spec = norm_model("f32", True)
    l = spec.stages[0].layers[1]
    for k, v in changed.items():
        setattr(l, k, v)
    with pytest.raises(eb.EEError):
        eb.EEModel(spec)


def test_silu_is_for_group_norm_alone():
    spec = norm_model("f32", True)
    spec.stages[0].layers[0].act = wl.ACT_SILU
    with pytest.raises(eb.EEError):
        eb.EEModel(spec)


# ----------------------------------------------------------------------------- calls behind one another

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("adapters", [0, 2])
def test_a_projection_whose_weight_the_call_before_it_writes(dtype, adapters):
    """weight = W2 (the first call's output), bias = probabilities (the second call's): both are there when they are read."""
    rows, c, n, rank = 4, 1024, 384, 8
    x, w, _, a, b, _, which = linear_operands(5, rows, c, n, rank, 2, dtype)
    inner = (normal(gen(6), c, 512) * 512 ** -0.5).to(TD[dtype])
    logits = normal(gen(7), 1, n)
    w2, bias, y = torch.zeros_like(w), torch.zeros((1, n), device="cuda"), torch.zeros((rows, n), dtype=TD[dtype], device="cuda")
    outer = (normal(gen(8), n, 512) * 512 ** -0.5).to(TD[dtype])
    ws = torch.empty(eb.adapted_linear_workspace_bytes(rows, rank), dtype=torch.uint8, device="cuda")

    def run():
        eb.adapted_linear(dtype, outer, n, 512, inner, c, None, None, 0, 0, None, w2, None)
        eb.softmax("f32", logits, 1, n, bias)
        eb.adapted_linear(dtype, x, rows, c, w2, n, a if adapters else None, b if adapters else None, rank, adapters, which if adapters else None, y,
                          ws if adapters else None, bias=bias)

    for times in range(5):
        w2.zero_(), bias.zero_(), y.zero_()
        run()
        linear_check(y, x, w2, bias[0], a[:adapters], b[:adapters], None, which, dtype)
        assert bool((w2 != 0).any())


# ----------------------------------------------------------------------------- at the ends of what they take

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_adapted_linear_of_the_most_rows(dtype):
    """2^22 rows: more blocks than the second and third dimension of a grid take."""
    rows, c, n = 1 << 22, 8, 1
    ops = linear_operands(3, rows, c, n, 2, 3, dtype)
    linear_run(dtype, ops)


@pytest.mark.parametrize("shape", [(300, 520, 4099, 24, 7), (700, 70, 5000, 16, 30), (700, 71, 5000, 3, 30), (290, 264, 9000, 5, 3)], ids=str)
def test_adapted_linear_of_more_tiles_than_processors(shape):
    linear_run("bf16", linear_operands(sum(shape), *shape, "bf16"))


@pytest.mark.parametrize("rows", [6, 200])
def test_adapted_linear_of_an_infinite_sum(rows):
    """a x is an infinity: the row is one, with the sign of b, and the others are not touched."""
    x, w, bias, a, b, scale, which = linear_operands(4, rows, 256, 130, 1, 2, "bf16")
    x, a = x.abs(), a.abs()
    b[b == 0] = 1.0
    scale[1] = float("inf")
    y, _ = out_like((rows, 130), torch.bfloat16)
    ws = torch.empty(eb.adapted_linear_workspace_bytes(rows, 1), dtype=torch.uint8, device="cuda")
    eb.adapted_linear("bf16", x, rows, 256, w, 130, a, b, 1, 2, which, y, ws, bias=bias, scale=scale)
    hit = which == 1
    assert bool(hit.any()) and torch.equal(y[hit], torch.copysign(torch.full_like(y[hit], float("inf")), b[1, :, 0].expand(int(hit.sum()), 130)))
    linear_check(y[~hit], x[~hit], w, bias, a, b, torch.ones_like(scale) * scale[0], torch.where(which == 1, -1, which)[~hit], "bf16")


@pytest.mark.parametrize("n", [70, 9000])
def test_verify_drafts_where_the_early_probabilities_are_infinite(n):
    p, q, d, u, r = drafts_of(n, 6, 2, n)
    q[0, :, 3::2], q[1, :, ::3], q[2] = -float("inf"), float("inf"), -float("inf")
    verify_case(p, q, d, u * 0 + 1 - 2.0 ** -24, r)
    verify_case(p, q, d, u, r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 500, 48, 8), (1, 20000, 48, 8), (3, 77, 64, 32), (1, 9000, 640, 64), (2, 300, 80, 4), (1, 30000, 64, 16), (1, 25001, 24, 12), (4, 6, 96, 16), (1, 40000, 40, 8)], ids=str)
def test_group_norm_of_groups_that_share_accesses(shape, dtype):
    """Groups of 2, 4, 5, 6, 10 and 20 channels: a 16-byte access holds two, four or eight runs of one group each, on maps that stay and that are read twice."""
    b, hw, c, groups = shape
    g = gen(sum(shape))
    x = (normal(g, b, hw, c) * (0.5 + normal(g, c).abs()) + 2 * normal(g, c)).to(TD[dtype])
    gamma, beta, res = 1 + 0.3 * normal(g, c), 0.5 * normal(g, c), normal(g, b, hw, c).to(TD[dtype])
    for act, residual in ((3, None), (1, res)):
        y, raw = out_like(x.shape, TD[dtype])
        eb.group_norm(dtype, x, b, hw, c, groups, gamma, beta, 1e-5, act, y, residual=residual)
        norm_check(y, x, gamma, beta, groups, 1e-5, act, dtype, residual)
        assert untouched(raw, 0, x.numel())
    eb.operators_check()


@pytest.mark.parametrize("order", ["mixed", "runs", "none", "one"])
@pytest.mark.parametrize("shape", [(300, 2048, 200, 64, 12), (300, 2050, 130, 64, 9), (200, 2047, 77, 70, 12), (700, 1024, 64, 128, 20), (130, 3600, 300, 57, 130), (1500, 4096, 260, 8, 40)], ids=str)
def test_adapted_linear_of_much_work_for_the_adapters(shape, order):
    """a x on the tensor cores: groups of adapters that fill a tile, side by side and one after the other."""
    linear_run("bf16", linear_operands(sum(shape), *shape, "bf16", order))


def test_adapted_linear_of_much_work_keeps_other_rows_out_of_a_row():
    rows, c, n, rank, adapters = 400, 2048, 260, 48, 9
    x, w, bias, a, b, scale, which = linear_operands(8, rows, c, n, rank, adapters, "bf16")
    y = linear_run("bf16", (x, w, bias, a, b, scale, which))
    x, a, b = x.clone(), a.clone(), b.clone()
    a[2], b[1], x[77] = float("nan"), float("inf"), float("inf")
    bad, _ = out_like(y.shape, torch.bfloat16)
    ws = torch.empty(eb.adapted_linear_workspace_bytes(rows, rank), dtype=torch.uint8, device="cuda")
    eb.adapted_linear("bf16", x, rows, c, w, n, a, b, rank, adapters, which, bad, ws, bias=bias, scale=scale)
    clean = (which != 1) & (which != 2)
    clean[77] = False
    assert torch.equal(bad[clean], y[clean]) and bool(bad[which == 2].isnan().all()) and bool((~bad[which == 1].isfinite()).all())
    eb.operators_check()
