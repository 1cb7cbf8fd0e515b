"""What ee.h promises of the operators that need no model, where a plain comparison of results does not look: calls from several host threads, values at the ends
of their types, statistics of extreme maps, what a row may depend on."""
import ctypes as C
import subprocess

import numpy as np
import pytest
import torch

from paper_2209_13443_b200 import binding as eb
from paper_2209_13443_b200 import workloads as wl
from tests.test_gpu_operators import TD, U, drafts_of, gen, linear_operands, linear_run, norm_check, norm_exact, normal, out_like, untouched

pytestmark = pytest.mark.gpu

# ----------------------------------------------------------------------------- several host threads

HAMMER = r"""
#include <thread>
typedef int (*softmax_fn)(int, const void*, int, int, const float*, float*, void*);
typedef int (*norm_fn)(int, const void*, const void*, int, int, int, int, const float*, const float*, float, int, void*, void*);
struct Work { const void* x; void* y; int n; void* stream; };
// Two host threads, each with calls of its own size on a stream of its own; returns how many calls failed.
template <typename F>
static int both(F call, const Work* w, int times) {
  int bad[2] = {0, 0};
  std::thread t[2];
  for (int i = 0; i < 2; ++i)
    t[i] = std::thread([=, &bad] {
      for (int k = 0; k < times; ++k) bad[i] += call(w[i]) != 0;
    });
  for (auto& x : t) x.join();
  return bad[0] + bad[1];
}
extern "C" int hammer_softmax(void* f, const Work* w, int times) {
  return both([f](const Work& k) { return ((softmax_fn)f)(0, k.x, 1, k.n, nullptr, (float*)k.y, k.stream); }, w, times);
}
extern "C" int hammer_norm(void* f, const Work* w, int times) {
  return both([f](const Work& k) { return ((norm_fn)f)(0, k.x, nullptr, 1, k.n, 32, 1, nullptr, nullptr, 1e-5f, 0, k.y, k.stream); }, w, times);
}
"""


class Work(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("n", C.c_int), ("stream", C.c_void_p)]


@pytest.mark.parametrize("op,sizes", [("softmax", (600000, 128001)), ("norm", (3500, 3200))])
def test_two_host_threads_with_calls_of_different_sizes(op, sizes, tmp_path):
    """Two lengths of a row, two sizes of a map, of one kernel, both beyond the 48 KB of shared memory that a launch has without asking."""
    src, so = tmp_path / "hammer.cpp", tmp_path / "hammer.so"
    src.write_text(HAMMER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-pthread", "-o", str(so), str(src)], check=True)
    width = 1 if op == "softmax" else 32
    xs = [normal(gen(n), n * width) for n in sizes]
    ys = [torch.empty_like(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in sizes]

    def alone(x, n):
        y = torch.empty_like(x)
        if op == "softmax":
            eb.softmax("f32", x, 1, n, y)
        else:
            eb.group_norm("f32", x, 1, n, 32, 1, None, None, 1e-5, 0, y)
        return y

    want = [alone(x, n) for x, n in zip(xs, sizes)]
    torch.cuda.synchronize()
    work = (Work * 2)(*[Work(x.data_ptr(), y.data_ptr(), n, s.cuda_stream) for x, y, n, s in zip(xs, ys, sizes, streams)])
    lib = eb.load_library()
    entry = C.cast(lib.ee_softmax if op == "softmax" else lib.ee_group_norm, C.c_void_p)
    failed = getattr(C.CDLL(str(so)), "hammer_" + op)(entry, work, 4000)
    torch.cuda.synchronize()
    assert failed == 0, f"{failed} of 8000 calls failed"
    assert all(torch.equal(a, b) for a, b in zip(ys, want))


# ----------------------------------------------------------------------------- softmax at the ends of its types

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [40, 900, 5000, 70001])
@pytest.mark.parametrize("t", [float("inf"), 3.4e38, 1.5e38, 1e38, 2e37, 1e36])
def test_softmax_so_hot_that_the_lowest_values_count(dtype, n, t):
    """Masks of the type's lowest value are numbers: at temperatures of their size they weigh what the formula says, infinities as masks still nothing.  Tolerance: that of
    (l - max) / t and of its power as ever (5 u of it + 52 u + the sum's chain of n / 512), and of a factor that is a subnormal number half its step, 2^-150, of
    at most 3.4e38 halves: 2.8 u, 5.6 u where t is infinite; each twice, for the value and for the sum."""
    inf, low = float("inf"), torch.finfo(TD[dtype]).min
    x = normal(gen(n), 5, n).to(TD[dtype])
    x[0, 7:] = low
    x[1, 5:] = -inf
    x[2], x[2, ::2] = low, -low                            # further apart than the type's largest value
    x[3, 3:9], x[3, 9:] = low, -inf
    x[4] = low
    y, raw = out_like((5, n), torch.float32)
    eb.softmax(dtype, x, 5, n, y, temperature=torch.full((5,), t, device="cuda"))
    z = x.double()
    d = (z.amax(1, keepdim=True) - z) / torch.tensor(t, device="cuda").double()       # finite / inf = 0
    d = torch.where(z == -inf, torch.full_like(d, inf), d)
    e = torch.exp(-d)
    ref = e / e.sum(1, keepdim=True)
    tol = ref * U * (5 * torch.where(d < 200, d, torch.zeros_like(d)) + 52 + n / 512 + 11.2) + 2.0 ** -126
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), f"off by {float((err / tol).max()):.3g} tolerances"
    assert bool((y[x == -inf] == 0).all()) and untouched(raw, 0, 5 * n)


# ----------------------------------------------------------------------------- adapted projection

@pytest.mark.parametrize("rows,c,rank", [(3, 8, 1), (100, 8, 1), (300, 4096, 48)])
@pytest.mark.parametrize("scale", [3.4e38, -3.4e38, 3.395e38])
def test_adapted_linear_of_the_largest_finite_sums(rows, c, rank, scale):
    """scale * a x is a float above the largest bf16: its two bf16 parts are that and the remainder, not an infinity.  b brings it back, so y = scale * 2^-127: off by 2^-17 of it for
    the two parts and half a step of bf16."""
    n = 16
    x, w, a, b = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((rows, c), (n, c), (1, rank, c), (1, n, rank)))
    x[:, 0], a[0, rank - 1, 0] = 1.0, 1.0
    b[0, :, rank - 1] = 2.0 ** -127
    y, raw = out_like((rows, n), torch.bfloat16)
    ws = torch.empty(eb.adapted_linear_workspace_bytes(rows, rank) + 256, dtype=torch.uint8, device="cuda")
    which = torch.zeros(rows, dtype=torch.int32, device="cuda")
    eb.adapted_linear("bf16", x, rows, c, w, n, a, b, rank, 1, which, y, ws, scale=torch.tensor([scale], device="cuda"))
    want = float(torch.tensor(scale, dtype=torch.float32)) * 2.0 ** -127
    assert bool(((y.double() - want).abs() <= abs(want) * (2.0 ** -17 + 2.0 ** -8)).all()) and untouched(raw, 0, rows * n)


@pytest.mark.parametrize("shape", [(300, 64, 40, 5), (9, 1001, 300, 3)], ids=str)
def test_adapted_linear_f32_rounds_the_scaled_sum_once(shape):
    """Rank 1, b = 1 and no shared weight leave y = scale * a x rounded to fp32.  The sum itself is off by c 2^-53 of its magnitudes, so one value in 2^29 / c, times what cancels in it,
    could round the other way: none of the few hundred here, and of c = 1001 at most one."""
    rows, c, n, m = shape
    x, w, _, a, b, scale, which = linear_operands(1, rows, c, n, 1, m, "f32")
    w, b = torch.zeros_like(w), torch.ones_like(b)
    y, raw = out_like((rows, n), torch.float32)
    ws = torch.empty(eb.adapted_linear_workspace_bytes(rows, 1) + 256, dtype=torch.uint8, device="cuda")
    eb.adapted_linear("f32", x, rows, c, w, n, a, b, 1, m, which, y, ws, scale=scale)
    at = which.long().clamp(min=0)
    want = torch.where(which >= 0, (x.double() * a[at, 0].double()).sum(1) * scale[at].double(), torch.zeros(rows, dtype=torch.float64, device="cuda")).float()
    assert int((y[:, 0] != want).sum()) <= (1 if c > 1000 else 0) and torch.equal(y, y[:, :1].expand_as(y)) and untouched(raw, 0, rows * n)


@pytest.mark.parametrize("shape", [(64, 4096, 512, 16, 32), (300, 520, 4099, 24, 7), (20, 512, 256, 5, 4), (256, 4096, 1024, 64, 9), (200, 2047, 300, 8, 12)], ids=str)
def test_adapted_linear_of_rows_beside_others_adapters(shape):
    """Half of the rows keep their adapters while the other half change theirs, and while the pool of adapters grows.  Rows without one keep their bits, the others what the
    order of a sum in fp32 moves: each call's values are within linear_check's bound (linear_run), so two calls' within twice that, the roundings to bf16 included."""
    rows, c, n, rank, m = shape
    x, w, bias, a, b, scale, which = linear_operands(8, *shape, "bf16")
    which[::8] = -1
    keep = torch.arange(rows, device="cuda") % 2 == 0
    first = linear_run("bf16", (x, w, bias, a, b, scale, which))
    has, none = keep & (which >= 0), keep & (which < 0)
    assert bool(has.any()) and bool(none.any())
    for seed in range(3):
        others = torch.randint(-1, m, (rows,), generator=gen(seed), device="cuda").int()
        changed = torch.where(keep, which, others)
        if seed == 2:
            a, b, scale = (torch.cat([t, torch.zeros((40,) + t.shape[1:], dtype=t.dtype, device="cuda")]) for t in (a, b, scale))
        y = linear_run("bf16", (x, w, bias, a, b, scale, changed))
        assert torch.equal(y[none], first[none])
        mag = x.double().abs() @ w.double().abs().t() + bias.double().abs()
        at = which.long().clamp(min=0)
        h = torch.bmm(a[at].double().abs(), x.double().abs()[:, :, None])
        share = torch.bmm(b[at].double().abs(), h)[:, :, 0] * scale[at, None].double()
        lost = (c / 16 + 20) * 2 * U * (mag + 2 * share) + 2.0 ** -17 * share
        off = (y.double() - first.double()).abs()
        assert bool((off <= 2 * (lost + 2.0 ** -8 * (first.double().abs() + lost)))[has].all())


# ----------------------------------------------------------------------------- group norm of groups that hardly vary, and of lone extremes

FLAT = [(2, 40, 16, 4), (3, 957, 96, 32), (1, 12544, 96, 8), (1, 60001, 64, 4), (2, 9, 1001, 1), (1, 20000, 3, 1), (1, 30, 6006, 1), (1, 10, 4096, 1), (1, 30000, 520, 40), (2, 3136, 64, 64), (3, 100, 30, 30)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", FLAT, ids=str)
def test_group_norm_of_constant_groups_is_beta(shape, dtype):
    """x - mean is 0 in every value, so the result is beta and nothing else, however large the constant and however small eps."""
    b, hw, c, groups = shape
    beta = normal(gen(2), c)
    y, raw = out_like((b, hw, c), TD[dtype])
    for value in (1000.0, 3008.0, 100.0, 0.3, -7e6):
        x = torch.full((b, hw, c), value, device="cuda").to(TD[dtype])
        for eps in (1e-5, 1e-12):
            eb.group_norm(dtype, x, b, hw, c, groups, None, beta, eps, 0, y)
            assert torch.equal(y, beta.to(TD[dtype]).expand_as(y)), (value, eps, float((y.float() - beta).abs().max()))
    assert untouched(raw, 0, x.numel())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", FLAT, ids=str)
def test_group_norm_of_groups_that_hardly_vary(shape, dtype):
    """Some values one step of bf16 above the others."""
    b, hw, c, groups = shape
    x = torch.full((b, hw, c), 1000.0, device="cuda")
    x[torch.rand((b, hw, c), generator=gen(4), device="cuda") < 0.02] = 1004.0
    x = x.to(TD[dtype])
    y, _ = out_like(x.shape, TD[dtype])
    eb.group_norm(dtype, x, b, hw, c, groups, None, None, 1e-5, 0, y)
    norm_check(y, x, None, None, groups, 1e-5, 0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1 << 20, 64, 8), (1, 1 << 18, 64, 1), (1, 50176, 32, 4), (1, 90000, 37, 1), (2, 2401, 37, 1), (1, 100003, 24, 8), (1, 70000, 64, 64), (1, 12544, 4096, 2)], ids=str)
def test_group_norm_of_one_extreme_pixel(shape, dtype):
    """A map of zeros but for its first pixel, of 10000: all differences but one are alike, and extreme, where they are taken from the first value.  A run of r accesses
    of V values, in four chains (one where V = 1), loses up to (r V)^2 / 8 u (r^2 / 2 u) of the mean and of the squares of its thread: with V = 4, r = 16 (fp32) and V = 1, r = 32
    512 u, with V = 8, r = 32 (bf16) 8192 u; half of the squares' goes into the deviation.  The sums of up to 300 later runs lose r V / 4 k u (r / k u) of the mean in the k-th
    (ln 300 + 1 < 7 of them), and its rounding one u each; the joins of threads, warps and CTAs below 100 u."""
    b, hw, c, groups = shape
    x = torch.zeros(b, hw, c, device="cuda")
    x[:, 0] = 1e4
    x = x.to(TD[dtype])
    y, _ = out_like(x.shape, TD[dtype])
    eb.group_norm(dtype, x, b, hw, c, groups, None, None, 1e-5, 0, y)
    ref = norm_exact(x, None, None, groups, 1e-5, 0)[0]
    lost = (1.5 * (512 if dtype == "f32" else 8192) + 7 * 64 + 300 + 100) * U
    tol = ref.abs() * (lost + (0 if dtype == "f32" else 2.0 ** -8 * (1 + lost))) + U * 1e-3
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), f"off by {float((err / tol).max()):.3g} tolerances"


@pytest.mark.parametrize("offset", [100.0, -3000.0, 1e5])
@pytest.mark.parametrize("residual", [False, True])
def test_group_norm_keeps_the_digits_below_a_large_mean(offset, residual):
    """fp32, a mean of thousands of deviations.  Differences from a value (or mean) nearby are exact, so the mean is rounded once in each join: threads, warps, CTAs, cluster: 4 u of
    it, and what its parts' roundings do to the squares between the parts is at most 2 u |mean| / deviation of them where a part's mean lies within half a deviation.  Sums
    of differences: chains of 12 accesses, four lanes, eight warps and CTAs, below 512 u of the deviation."""
    b, hw, c, groups = 2, 3000, 32, 2
    g = gen(9)
    x = normal(g, b, hw, c) + offset
    res = normal(g, b, hw, c) if residual else None
    y, _ = out_like(x.shape, torch.float32)
    eb.group_norm("f32", x, b, hw, c, groups, None, None, 1e-5, 0, y, residual=res)
    ref, t, z, mean, var = norm_exact(x, None, None, groups, 1e-5, 0, res)
    far = (mean.abs() / torch.sqrt(var)).expand(b, hw, groups, c // groups).reshape(b, hw, c) + z.abs()
    tol = U * far * (4.5 + z.abs()) + 512 * U * (1 + z.abs()) + 4 * U * ref.abs()
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), f"off by {float((err / tol).max()):.3g} tolerances"


# ----------------------------------------------------------------------------- waits that run out

def _late(call, outs):
    """`call` with a limit of one clock on the waits between the blocks of a cluster, until a wait has run out (a block that happens to be its cluster's last has nothing to wait
    for), from outputs filled with 77; then with the limit back.  What a block that gave up left is 77, everything else right."""
    for o in outs:
        o.fill_(77)
    call()
    eb.operators_check()
    want = [o.clone() for o in outs]
    eb.operators_set_wait_limit(1)
    try:
        seen = False
        for _ in range(20):
            for o in outs:
                o.fill_(77)
            call()
            torch.cuda.synchronize()
            try:
                eb.operators_check()
            except eb.EEError as e:
                assert e.status == 7                                   # EE_ERR_TIMEOUT
                seen = True
            for o, w in zip(outs, want):
                assert bool(((o == w) | (o == 77)).all())
            if seen:
                break
        assert seen
    finally:
        eb.operators_set_wait_limit(4_000_000_000)
    for o in outs:
        o.fill_(77)
    call()
    eb.operators_check()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def _whatever_the_limit(call, outs):
    """`call` under limits from far too short to long enough, a tenth apart.  Between them the own products of some blocks come in time and those of others do not: whoever lacks a part of its sums leaves
    its outputs (77) as they are."""
    for o in outs:
        o.fill_(77)
    call()
    eb.operators_check()
    want, late = [o.clone() for o in outs], 0
    try:
        for step in range(62):
            eb.operators_set_wait_limit(int(100 * 1.1 ** step))
            for _ in range(6):
                for o in outs:
                    o.fill_(77)
                call()
                try:
                    eb.operators_check()
                except eb.EEError as e:
                    assert e.status == 7                               # EE_ERR_TIMEOUT
                    late += 1
                for o, w in zip(outs, want):
                    assert bool(((o == w) | (o == 77)).all())
    finally:
        eb.operators_set_wait_limit(4_000_000_000)
    assert late
    for o in outs:
        o.fill_(77)
    call()
    eb.operators_check()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 3136, 64, 8), (1, 30000, 520, 40), (3, 957, 96, 32)], ids=str)
def test_group_norm_whose_exchange_runs_out_of_time(shape, dtype):
    b, hw, c, groups = shape
    x = normal(gen(1), b, hw, c).to(TD[dtype])
    y = torch.empty_like(x)
    _late(lambda: eb.group_norm(dtype, x, b, hw, c, groups, None, None, 1e-5, 3, y), [y])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [32769, 128001, 614399])
def test_softmax_whose_exchange_runs_out_of_time(n, dtype):
    x, y = normal(gen(n), 3, n).to(TD[dtype]), torch.empty((3, n), device="cuda")
    for heat in (None, torch.zeros(3, device="cuda")):
        _late(lambda: eb.softmax(dtype, x, 3, n, y, temperature=heat), [y])


@pytest.mark.parametrize("dtype,shape", [("bf16", (1, 2048, 1000, 8, 16)), ("bf16", (64, 4096, 512, 16, 32)), ("bf16", (40, 1001, 300, 3, 4)), ("bf16", (256, 4096, 256, 64, 9)), ("f32", (37, 2048, 1000, 5, 7))], ids=str)
def test_adapted_linear_whose_exchange_runs_out_of_time(dtype, shape):
    rows, c, n, rank, m = shape
    x, w, bias, a, b, scale, which = linear_operands(2, *shape, dtype)
    y, ws = torch.empty((rows, n), dtype=TD[dtype], device="cuda"), torch.empty(eb.adapted_linear_workspace_bytes(rows, rank) + 256, dtype=torch.uint8, device="cuda")
    _late(lambda: eb.adapted_linear(dtype, x, rows, c, w, n, a, b, rank, m, which, y, ws, bias=bias, scale=scale), [y])


@pytest.mark.parametrize("n", [20001, 128001])
def test_verify_drafts_whose_exchange_runs_out_of_time(n):
    p, q, d, u, r = drafts_of(n, 9, 3, n)
    p[3], q[4, 0] = 0.0, 2.0                               # a second round: p - q leaves nothing
    tokens, accepted = torch.empty((9, 4), dtype=torch.int32, device="cuda"), torch.empty(9, dtype=torch.int32, device="cuda")
    _late(lambda: eb.verify_drafts(p, q, d, u, r, 9, 3, n, tokens, accepted), [tokens, accepted])


def test_a_models_group_norms_go_by_its_limit():
    """As its other layers do: with a limit of one clock the wait for a cluster's statistics runs out and is reported once."""
    spec = wl.Model("norm", "bf16", 256, 256, 64, [wl.Stage([wl.Layer(wl.OP_GROUPNORM, 64, 64, act=wl.ACT_RELU, norm_groups=8, norm_eps=1e-5)], 10, np.zeros((10, 64), np.float32),
                                                           np.zeros(10, np.float32), 0.0, True)], 2)
    m = eb.EEModel(spec)
    ws = m.workspace()
    x = normal(gen(0), 2, 256, 256, 64).to(torch.bfloat16)
    y, want = torch.full_like(x, 77), torch.empty_like(x)
    m.layer_run(0, 0, x, None, 2, want, ws)
    m.check()
    m.set_wait_limit(1)
    m.layer_run(0, 0, x, None, 2, y, ws)
    with pytest.raises(eb.EEError) as e:
        m.check()
    assert e.value.status == 7 and bool(((y == want) | (y == 77)).all())
    m.set_wait_limit(4_000_000_000)
    m.layer_run(0, 0, x, None, 2, y, ws)
    m.check()
    assert torch.equal(y, want)
    m.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,n", [(1, 2048, 1000), (3, 8192, 512), (16, 4096, 2048), (40, 8199, 300), (128, 2048, 256)])
def test_int8_linear_in_which_some_products_are_late(rows, c, n, dtype):
    g = gen(rows + c)
    x = normal(g, rows, c).to(TD[dtype])
    w = torch.zeros(n, eb.int8_row_bytes(c), dtype=torch.int8, device="cuda")
    w[:, :c] = torch.randint(-127, 128, (n, c), generator=g, device="cuda")
    y, room = torch.empty(rows, n, dtype=TD[dtype], device="cuda"), torch.empty(eb.int8_linear_workspace_bytes(rows, c) + 256, dtype=torch.uint8, device="cuda")
    _whatever_the_limit(lambda: eb.int8_linear(dtype, x, rows, c, w, None, n, y, workspace=room), [y])


@pytest.mark.parametrize("shape", [(1, 2048, 1000, 8, 16), (16, 8192, 512, 16, 32), (64, 4096, 512, 16, 32), (40, 1001, 300, 3, 4), (256, 4096, 256, 64, 9)], ids=str)
def test_adapted_linear_in_which_some_products_are_late(shape):
    rows, c, n, rank, m = shape
    x, w, bias, a, b, scale, which = linear_operands(3, *shape, "bf16")
    y, ws = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda"), torch.empty(eb.adapted_linear_workspace_bytes(rows, rank) + 256, dtype=torch.uint8, device="cuda")
    _whatever_the_limit(lambda: eb.adapted_linear("bf16", x, rows, c, w, n, a, b, rank, m, which, y, ws, bias=bias, scale=scale), [y])


def test_adapted_linear_of_nan_in_every_bit():
    """Sums of products with NaN of any bits are NaN, in a tile whose K a cluster shares."""
    rows, c, n, rank, m = shape = (20, 4096, 300, 4, 3)
    x, w, bias, a, b, scale, which = linear_operands(4, *shape, "bf16")
    bits = torch.tensor([-1, 0x7fff, 0x7fc0, -64, 0x7f81, -127], dtype=torch.int16, device="cuda")      # 0xffff, 0x7fff, 0x7fc0, 0xffc0, 0x7f81, 0xff81
    for i in range(6):
        x[2 * i, 700 * i] = bits[i:i + 1].view(torch.bfloat16)[0]
    w[7, 5], w[9, 4000] = bits[:1].view(torch.bfloat16)[0], bits[3:4].view(torch.bfloat16)[0]
    y, ws = torch.full((rows, n), 77, dtype=torch.bfloat16, device="cuda"), torch.empty(eb.adapted_linear_workspace_bytes(rows, rank) + 256, dtype=torch.uint8, device="cuda")
    eb.adapted_linear("bf16", x, rows, c, w, n, a, b, rank, m, which, y, ws, bias=bias, scale=scale)
    eb.operators_check()
    bad = torch.zeros(rows, n, dtype=torch.bool, device="cuda")
    bad[[0, 2, 4, 6, 8, 10]] = True
    bad[:, [7, 9]] = True
    assert torch.equal(y.isnan(), bad) and not bool((y == 77).any())
