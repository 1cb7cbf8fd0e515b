"""Refusals of the operators for rows in 8 bits and for drawn answers: they come before anything touches a device, so they are checked without one."""
import ctypes as C
import os
import re

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


QUANT = dict(dtype=BF16, x=P[0], rows=3, c=20, q=P[1], scale=P[2], stream=None)


@pytest.mark.parametrize("changed", [dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(c=0), dict(x=None), dict(q=None), dict(scale=None), dict(x=P[0] + 1), dict(q=P[1] + 8), dict(scale=P[2] + 2),
                                     dict(dtype=F32, x=P[0] + 2), dict(q=P[0]), dict(q=P[0] + 112), dict(scale=P[0] + 116), dict(scale=P[1] + 92), dict(x=P[1] + 94)])
def test_quantize_rows_refuses(changed):
    assert call("ee_quantize_rows", QUANT, **changed) == INVALID


def test_quantize_rows_of_nothing_and_of_too_much():
    assert call("ee_quantize_rows", QUANT, rows=0, x=None, q=None, scale=None) == 0
    assert call("ee_quantize_rows", QUANT, c=131072) == CAPACITY


def test_bytes_of_a_row():
    lib = eb.load_library()
    assert [lib.ee_int8_row_bytes(c) for c in (-1, 0, 1, 15, 16, 17, 4096, 131071, 131072)] == [0, 0, 16, 16, 16, 32, 4096, 131072, 0]


READ = dict(dtype=BF16, q=P[0], scale=P[1], pool=5, c=20, index=P[2], rows=3, y=P[3], stream=None)


@pytest.mark.parametrize("changed", [dict(dtype=2), dict(rows=-1), dict(pool=-1), dict(c=0), dict(index=None, pool=2), dict(q=None), dict(scale=None), dict(y=None), dict(q=P[0] + 4), dict(scale=P[1] + 2),
                                     dict(index=P[2] + 2), dict(y=P[3] + 1), dict(dtype=F32, y=P[3] + 2), dict(y=P[0]), dict(y=P[0] + 158), dict(y=P[1] + 18), dict(y=P[2] + 10), dict(index=P[3] + 116)])
def test_dequantize_rows_refuses(changed):
    assert call("ee_dequantize_rows", READ, **changed) == INVALID


def test_dequantize_rows_of_nothing_and_of_too_much():
    assert call("ee_dequantize_rows", READ, rows=0, q=None, scale=None, y=None) == 0
    assert call("ee_dequantize_rows", READ, pool=0, q=None, scale=None, y=None) == 0       # every index is outside: nothing is written
    assert call("ee_dequantize_rows", READ, c=131072) == CAPACITY


LINEAR = dict(dtype=BF16, x=P[0], x_scale=None, rows=5, c=40, weight=P[1], weight_scale=P[2], n=30, bias=P[3], y=P[4], workspace=P[5], workspace_bytes=1 << 20, stream=None)
GIVEN = dict(LINEAR, x_scale=P[6], workspace=None, workspace_bytes=0)


@pytest.mark.parametrize("changed", [dict(dtype=2), dict(rows=-1), dict(c=0), dict(n=0), dict(x=None), dict(weight=None), dict(y=None), dict(workspace=None), dict(workspace=P[5] + 128), dict(x=P[0] + 1),
                                     dict(weight=P[1] + 8), dict(weight_scale=P[2] + 2), dict(bias=P[3] + 1), dict(y=P[4] + 1), dict(y=P[0] + 398), dict(y=P[1]), dict(y=P[2] + 116), dict(y=P[3]),
                                     dict(y=P[5]), dict(y=P[5] + 256 + 18), dict(workspace=P[0]), dict(workspace=P[1] + 256), dict(workspace=P[2]), dict(workspace=P[3])])
def test_int8_linear_refuses(changed):
    assert call("ee_int8_linear", LINEAR, **changed) == INVALID


@pytest.mark.parametrize("changed", [dict(x=P[0] + 8), dict(x_scale=P[6] + 2), dict(y=P[0] + 238), dict(y=P[6] + 18), dict(weight=P[4]), dict(bias=P[4] + 296)])
def test_int8_linear_refuses_of_quantised_rows(changed):
    assert call("ee_int8_linear", GIVEN, **changed) == INVALID


def test_int8_linear_workspace():
    lib = eb.load_library()
    assert lib.ee_int8_linear_workspace_bytes(5, 40) == 256 + 20
    assert [lib.ee_int8_linear_workspace_bytes(*a) for a in ((0, 40), (-1, 40), (5, 0), (5, 131072))] == [0, 0, 0, 0]
    assert lib.ee_int8_linear_workspace_bytes(1 << 22, 131071) == (1 << 39) + (1 << 24)
    assert call("ee_int8_linear", LINEAR, workspace_bytes=275) == CAPACITY
    assert call("ee_int8_linear", LINEAR, rows=(1 << 22) + 1) == CAPACITY
    assert call("ee_int8_linear", LINEAR, n=(1 << 20) + 1) == CAPACITY
    assert call("ee_int8_linear", LINEAR, c=131072) == CAPACITY
    assert call("ee_int8_linear", LINEAR, rows=0, x=None, weight=None, y=None) == 0


SAMPLE = dict(dtype=F32, logits=P[0], rows=3, n=100, temperature=P[1], top_k=P[2], top_p=P[3], min_p=P[4], u=P[5], tokens=P[6], probs=P[7], stream=None)


@pytest.mark.parametrize("changed", [dict(dtype=2), dict(rows=-1), dict(n=0), dict(logits=None), dict(tokens=None, probs=None), dict(u=None), dict(logits=P[0] + 2), dict(temperature=P[1] + 1), dict(top_k=P[2] + 2),
                                     dict(top_p=P[3] + 3), dict(min_p=P[4] + 2), dict(u=P[5] + 1), dict(tokens=P[6] + 2), dict(probs=P[7] + 2), dict(probs=P[0] + 4), dict(dtype=BF16, probs=P[0]),
                                     dict(tokens=P[0] + 1196), dict(tokens=P[1] + 8), dict(tokens=P[2]), dict(tokens=P[3]), dict(tokens=P[4]), dict(tokens=P[5]), dict(tokens=P[7] + 1196), dict(probs=P[1]),
                                     dict(top_k=P[7]), dict(top_p=P[7] + 400), dict(min_p=P[7] + 1196), dict(u=P[7])])
def test_sample_refuses(changed):
    assert call("ee_sample", SAMPLE, **changed) == INVALID


def test_sample_of_nothing_and_of_too_much():
    assert call("ee_sample", SAMPLE, rows=0, logits=None, tokens=None, probs=None) == 0
    assert call("ee_sample", SAMPLE, n=614401) == CAPACITY
    assert call("ee_sample", SAMPLE, rows=2 ** 28, n=9, logits=1 << 50, probs=1 << 60) == CAPACITY


def test_prototypes_match_the_header():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "ee.h")).read(), flags=re.S)
    lib = eb.load_library()
    for name in ("ee_quantize_rows", "ee_int8_row_bytes", "ee_dequantize_rows", "ee_int8_linear", "ee_int8_linear_workspace_bytes", "ee_sample"):
        decl = re.search(r"\b" + name + r"\s*\((.*?)\)\s*;", src, flags=re.S).group(1)
        want = [C.c_void_p if "*" in a else C.c_float if "float" in a else C.c_size_t if "size_t" in a else C.c_int for a in decl.split(",")]
        assert getattr(lib, name).argtypes == want, name


CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2209_13443_b200", "csrc")
KERNELS = r"__global__ void[^;{]*?\n(\w+)\(([^{]*?)\) \{(.*?)\n\}\n"


def test_what_a_launch_in_front_may_write_is_not_declared_read_only():
    """As in the other operators: a kernel that starts before the one in front has ended does not promise that nobody writes its inputs."""
    seen = 0
    for name in ("quant.cuh", "sample.cuh"):
        for m in re.finditer(KERNELS, open(os.path.join(CSRC, name)).read(), flags=re.S):
            assert "griddepcontrol.wait" in m.group(3) and "__restrict__" not in m.group(2), m.group(1)
            seen += 1
    assert seen >= 5


def test_a_block_whose_wait_for_its_cluster_runs_out_stays_until_the_stores_to_it_have_landed():
    seen = 0
    for name in ("quant.cuh", "sample.cuh"):
        for m in re.finditer(KERNELS, open(os.path.join(CSRC, name)).read(), flags=re.S):
            if "mbar_wait_cluster(" in m.group(3):
                seen += 1
                assert "cluster_drain(" in m.group(3), m.group(1)
    assert seen >= 1
