"""Host side of qesgd_debug_matrix_plan: refusals, its words before and after calls that launch nothing, and its names."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def qesgd():
    from paper_1901_03040_b200 import build
    build.build()
    from paper_1901_03040_b200 import qesgd as mod
    return mod


def test_refusals(qesgd):
    plan = (C.c_uint32 * 8)()
    assert qesgd.lib.qesgd_debug_matrix_plan(None, plan) == qesgd.EINVAL
    assert qesgd.lib.qesgd_debug_matrix_plan(C.cast(C.create_string_buffer(4096), C.c_void_p), None) == qesgd.EINVAL


def test_a_call_that_fails_leaves_the_plan(qesgd):
    import torch
    if torch.cuda.is_available():
        pytest.skip("would run an accepted call on made-up addresses")
    ctx = C.cast(C.create_string_buffer(4096), C.c_void_p)      # zeros stand in for a context
    some = C.c_void_p(4096)
    assert qesgd.lib.qesgd_fp4_matmul(ctx, some, some, None, some, some, None, 10, 20, 30, 1, some, 0, 20, 0) == qesgd.ECUDA
    assert qesgd.lib.qesgd_fp4_matmul(ctx, some, some, None, some, some, None, 0, 20, 30, 1, some, 0, 20, 0) == qesgd.OK
    plan = (C.c_uint32 * 8)(*[7] * 8)
    assert qesgd.lib.qesgd_debug_matrix_plan(ctx, plan) == qesgd.OK and list(plan) == [0] * 8


def test_names_are_those_of_the_header(qesgd):
    text = open(os.path.join(ROOT, "include", "qesgd.h")).read()
    names = re.findall(r"#define QESGD_(MATRIX_\w+) (\d+)u", text)
    assert len(names) == 6
    for name, value in names:
        assert getattr(qesgd, name) == int(value)
