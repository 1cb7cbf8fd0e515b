"""Refusals of the operators that need no model: they come before anything touches a device, so they are checked without one."""
import ctypes as C

import pytest

from paper_2209_13443_b200 import binding as eb

INVALID, CAPACITY = eb.STATUS_NAMES.index("EE_ERR_INVALID_ARG"), eb.STATUS_NAMES.index("EE_ERR_CAPACITY")
P = [0x7f0000000000 + (i << 32) for i in range(12)]     # addresses far apart; nothing is read through them
F32, BF16 = 0, 1


def call(name, good, **changed):
    args = dict(good)
    for k, v in changed.items():
        assert k in args, k
        args[k] = v
    return getattr(eb.load_library(), name)(*args.values())


NORM = dict(dtype=F32, x=P[0], residual=P[1], batch=2, hw=9, c=12, groups=4, gamma=P[2], beta=P[3], eps=1e-5, act=1, y=P[4], stream=None)


@pytest.mark.parametrize("changed", [
    dict(dtype=2), dict(dtype=-1), dict(batch=-1), dict(hw=0), dict(c=0), dict(groups=0), dict(groups=5), dict(groups=24), dict(eps=-1e-9),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(act=-1), dict(act=4), dict(x=None), dict(y=None), dict(x=P[0] + 2), dict(y=P[4] + 1), dict(residual=P[1] + 2),
    dict(gamma=P[2] + 2), dict(beta=P[3] + 1), dict(y=P[0] + 4), dict(y=P[1] + 2 * 9 * 12 * 4 - 4), dict(dtype=BF16, x=P[0] + 1)])
def test_group_norm_refuses(changed):
    assert call("ee_group_norm", NORM, **changed) == INVALID


@pytest.mark.parametrize("changed", [dict(y=P[2]), dict(y=P[3]), dict(y=P[2] + 11 * 4), dict(gamma=P[4] + 2 * 9 * 12 * 4 - 4), dict(beta=P[4] - 11 * 4), dict(gamma=P[4] + 16), dict(beta=P[4])])
def test_group_norm_refuses_an_output_on_top_of_gamma_or_beta(changed):
    assert call("ee_group_norm", NORM, **changed) == INVALID


def test_group_norm_of_nothing_and_of_too_much():
    assert call("ee_group_norm", NORM, batch=0, x=None, y=None, residual=None) == 0
    # a slice a block at the least: 2^31 - 1 samples of two slices are more blocks than a grid has
    assert call("ee_group_norm", NORM, batch=2 ** 31 - 1, hw=256, c=256, groups=2, residual=None, x=1 << 50, y=1 << 60) == CAPACITY
    # a group of 2^22 pixels of 65521 odd rows: 2^35 loads of a block
    assert call("ee_group_norm", NORM, batch=1, hw=1 << 22, c=65521, groups=1, residual=None, x=1 << 50, y=1 << 60) == CAPACITY
    assert call("ee_group_norm", NORM, batch=2 ** 31 - 1, hw=2 ** 31 - 1, c=1, groups=1, residual=None, x=1 << 40, y=1 << 60) == CAPACITY


LINEAR = dict(dtype=BF16, x=P[0], rows=5, c=64, weight=P[1], n=40, bias=P[2], a=P[3], b=P[4], rank=8, n_adapters=3, scale=P[5], adapter=P[6], y=P[7], workspace=P[8],
              workspace_bytes=5 * 8 * 4, stream=None)


@pytest.mark.parametrize("changed", [
    dict(dtype=7), dict(rows=-1), dict(c=0), dict(n=0), dict(n_adapters=-1), dict(rank=0), dict(rank=129), dict(x=None), dict(weight=None), dict(y=None), dict(a=None), dict(b=None),
    dict(adapter=None), dict(workspace=None), dict(workspace=P[8] + 128), dict(x=P[0] + 1), dict(weight=P[1] + 1), dict(bias=P[2] + 2), dict(scale=P[5] + 2), dict(adapter=P[6] + 2),
    dict(y=P[0]), dict(y=P[0] + 5 * 64 * 2 - 2), dict(y=P[8]), dict(workspace=P[0]), dict(n_adapters=2 ** 30, rank=2)])
def test_adapted_linear_refuses(changed):
    assert call("ee_adapted_linear", LINEAR, **changed) == INVALID


def test_adapted_linear_workspace():
    lib = eb.load_library()
    assert lib.ee_adapted_linear_workspace_bytes(5, 8) == 5 * 8 * 4
    assert lib.ee_adapted_linear_workspace_bytes(0, 8) == 0 and lib.ee_adapted_linear_workspace_bytes(5, -1) == 0
    assert lib.ee_adapted_linear_workspace_bytes(1 << 22, 128) == 4 * 128 << 22
    assert call("ee_adapted_linear", LINEAR, workspace_bytes=5 * 8 * 4 - 1) == CAPACITY
    assert call("ee_adapted_linear", LINEAR, rows=(1 << 22) + 1) == CAPACITY
    assert call("ee_adapted_linear", LINEAR, rows=0, x=None, weight=None, y=None) == 0
    for size in ("c", "n"):
        assert call("ee_adapted_linear", LINEAR, **{size: (1 << 20) + 1}) == CAPACITY


@pytest.mark.parametrize("changed", [dict(y=P[1] + 40 * 64 * 2 - 2), dict(y=P[2] + 40 * 4 - 2), dict(y=P[3]), dict(y=P[4] + 3 * 40 * 8 * 2 - 2), dict(y=P[5]), dict(y=P[6] + 2), dict(workspace=P[1]),
                                     dict(workspace=P[2]), dict(workspace=P[3] + 256), dict(workspace=P[4]), dict(workspace=P[5]), dict(workspace=P[6])])
def test_adapted_linear_refuses_outputs_on_top_of_inputs(changed):
    assert call("ee_adapted_linear", LINEAR, **changed) == INVALID


SOFTMAX = dict(dtype=F32, logits=P[0], rows=3, n=100, temperature=P[1], probs=P[2], stream=None)


@pytest.mark.parametrize("changed", [dict(dtype=3), dict(rows=-1), dict(n=0), dict(logits=None), dict(probs=None), dict(logits=P[0] + 2), dict(probs=P[2] + 2), dict(temperature=P[1] + 1),
                                     dict(probs=P[0] + 4), dict(dtype=BF16, probs=P[0]), dict(temperature=P[2] + 1196)])
def test_softmax_refuses(changed):
    assert call("ee_softmax", SOFTMAX, **changed) == INVALID


def test_softmax_of_nothing_and_of_too_much():
    assert call("ee_softmax", SOFTMAX, rows=0, logits=None, probs=None) == 0
    assert call("ee_softmax", SOFTMAX, n=614401) == CAPACITY
    assert call("ee_softmax", SOFTMAX, rows=2 ** 28, n=9, logits=1 << 50, probs=1 << 60) == CAPACITY


VERIFY = dict(p=P[0], q=P[1], drafts=P[2], u=P[3], r=P[4], n_draft=P[5], batch=2, k=3, n=10, tokens=P[6], n_accepted=P[7], stream=None)


@pytest.mark.parametrize("changed", [dict(batch=-1), dict(k=-1), dict(n=0), dict(p=None), dict(r=None), dict(drafts=None), dict(u=None), dict(tokens=None), dict(n_accepted=None),
                                     dict(p=P[0] + 2), dict(q=P[1] + 1), dict(drafts=P[2] + 2), dict(u=P[3] + 2), dict(r=P[4] + 1), dict(n_draft=P[5] + 2), dict(tokens=P[6] + 2),
                                     dict(n_accepted=P[7] + 2)])
def test_verify_drafts_refuses(changed):
    assert call("ee_verify_drafts", VERIFY, **changed) == INVALID


@pytest.mark.parametrize("changed", [dict(tokens=P[0] + 2 * 4 * 10 * 4 - 4), dict(tokens=P[1]), dict(tokens=P[2]), dict(tokens=P[3] + 20), dict(tokens=P[4] + 4), dict(tokens=P[5]), dict(tokens=P[7] - 4),
                                     dict(n_accepted=P[2] + 20), dict(n_accepted=P[5]), dict(n_accepted=P[6] + 28)])
def test_verify_drafts_refuses_outputs_on_top_of_inputs(changed):
    assert call("ee_verify_drafts", VERIFY, **changed) == INVALID


def test_verify_drafts_of_nothing_and_of_too_much():
    assert call("ee_verify_drafts", VERIFY, batch=0, p=None, r=None) == 0
    assert call("ee_verify_drafts", VERIFY, batch=2 ** 31 - 1) == CAPACITY
    assert call("ee_verify_drafts", VERIFY, k=2 ** 31 - 1) == CAPACITY


@pytest.mark.parametrize("cycles", [0, -1, -2 ** 62])
def test_a_limit_of_the_waits_is_positive(cycles):
    assert eb.load_library().ee_operators_set_wait_limit(cycles) == INVALID


def test_prototypes_match_the_header():
    """As many arguments in the binding as in the header, pointers where it has pointers."""
    import os
    import re

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "ee.h")).read(), flags=re.S)
    lib = eb.load_library()
    for name in ("ee_group_norm", "ee_adapted_linear", "ee_adapted_linear_workspace_bytes", "ee_softmax", "ee_verify_drafts", "ee_operators_check"):
        decl = re.search(r"\b" + name + r"\s*\((.*?)\)\s*;", src, flags=re.S).group(1)
        want = [C.c_void_p if "*" in a else C.c_float if "float" in a else C.c_size_t if "size_t" in a else C.c_int for a in decl.split(",")]
        assert getattr(lib, name).argtypes == want, name


def test_what_a_launch_in_front_may_write_is_not_declared_read_only():
    """A kernel that starts before the one in front has ended must not promise (`__restrict__`) that nobody writes its inputs while it lives: such loads may be served by
    a cache that the wait for that kernel does not clear.  Operands that only the past of the stream writes may keep it."""
    import os
    import re

    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2209_13443_b200", "csrc")
    past = {"lowrank_delta_kernel": {"b", "which"}, "conv_igemm_f64mma_kernel": {"x", "w", "scale", "bias"}}     # of the former, a plain launch is in between; of the latter, x is only copied
    seen = 0
    for name in ("norm.cuh", "draft.cuh", "lowrank.cuh", "conv_f32.cuh"):
        src = open(os.path.join(csrc, name)).read()
        for m in re.finditer(r"__global__ void[^;{]*?\n(\w+)\(([^{]*?)\) \{(.*?)\n\}\n", src, flags=re.S):
            if "griddepcontrol.wait" not in m.group(3):
                continue
            seen += 1
            only = {re.search(r"(\w+)\s*$", a).group(1) for a in m.group(2).split(",") if "__restrict__" in a}
            assert only <= past.get(m.group(1), set()), (m.group(1), only)
    assert seen >= 6


def test_a_block_whose_wait_for_its_cluster_runs_out_stays_until_the_stores_to_it_have_landed():
    """Every kernel that waits for other CTAs' asynchronous stores meets them (cluster_drain) before it leaves without them: stores that land in the shared
    memory of a CTA that has gone are a fault."""
    import os
    import re

    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2209_13443_b200", "csrc")
    seen = 0
    for name in ("norm.cuh", "draft.cuh", "lowrank.cuh", "conv_f32.cuh", "head.cuh"):
        for m in re.finditer(r"__global__ void[^;{]*?\n(\w+)\([^{]*?\) \{(.*?)\n\}\n", open(os.path.join(csrc, name)).read(), flags=re.S):
            if "mbar_wait_cluster(" in m.group(2):
                seen += 1
                assert "cluster_drain(" in m.group(2), m.group(1)
    assert seen >= 6
