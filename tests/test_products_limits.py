"""Sizes at the ends of what the experts' products take, without a GPU: what the kernels' arithmetic cannot hold is refused."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import paper_2401_08383_amd as exf
from paper_2401_08383_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _p(i):  # aligned, never dereferenced
    return ctypes.c_void_p((i + 1) << 40)


ROWS = (1 << 31) - 1024  # EXF_MAX_PRODUCT_ROWS
CALLS = {  # the result is NULL: sizes that are taken come back with that error, and nothing is launched
    "product": lambda A, dt: exf.lib().moe_grouped_product(_p(0), _p(1), _p(2), None, A, 8, 8, 1, dt, None, None),
    "dx": lambda A, dt: exf.lib().moe_grouped_product_dx(_p(0), _p(1), _p(2), A, 8, 8, 1, dt, None, None),
    "dw": lambda A, dt: exf.lib().moe_grouped_product_dw(_p(0), _p(1), _p(2), A, 8, 8, 1, dt, dt, None, None, _p(3), 1 << 40, None),
    "mx4": lambda A, dt: exf.lib().moe_grouped_product_mx4(_p(0), _p(1), _p(2), _p(3), _p(4), None, A, 8, 32, 1, dt, None, None, 0, None),
}


@pytest.mark.parametrize("dt", [B.EXF_BF16, B.EXF_F32])
@pytest.mark.parametrize("call", list(CALLS))
def test_rows(call, dt):
    """An expert with all rows: they are rounded up to tiles of 320 rows and stages of 64 in 32 bits.  With 2^31 - 63 rows and more the weights'
    gradient had a negative number of stages, and came out as zeros."""
    for rows in (ROWS + 1, (1 << 31) - 64, (1 << 31) - 1):
        assert CALLS[call](rows, dt) == B.EXF_ERR_BAD_SHAPE, rows
    assert CALLS[call](ROWS, dt) == B.EXF_ERR_NULL_PTR
    int32 = lambda v: ctypes.c_int32(v).value  # noqa: E731
    assert int32((1 << 31) - 63 + 63) < 0  # what they were
    for step in (64, 320, 12 * 64):  # a stage, the tallest tile, the stages that small tiles look ahead
        assert int32(ROWS + step) == ROWS + step


# Sizes that no call takes, some of which overflow to zero on the way to a division.
@pytest.mark.parametrize("query", ["mx4_workspace_bytes(1 << 62, 64, 4)", "mx4_workspace_bytes(1 << 40, 1 << 30, 1 << 24)", "mx4_workspace_bytes(-1, 64, 32)",
                                   "dw_workspace_bytes(1000, 8, 8, 1 << 24, 0)", "dw_workspace_bytes(1000, 8, 8, 1 << 24, 1)", "dw_workspace_bytes(1 << 62, 2147483647, 8, 1, 0)",
                                   "dw_workspace_bytes(1 << 20, 64, 2147483647, 1, 1)", "dw_workspace_bytes(1 << 20, 64, 64, 65, 0)", "dw_workspace_bytes(1 << 20, 64, 64, 1, 7)"])
def test_queries_of_sizes_that_no_call_takes(query):
    code = f"import paper_2401_08383_amd as exf; assert exf.lib().moe_grouped_product_{query} == 0"
    assert subprocess.run([sys.executable, "-c", code], cwd=ROOT).returncode == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="what fails here is that there is no GPU")
def test_errors_name_the_call():
    """bf16 with few rows an expert goes to the weight streams, whose other user is moe_expert_ffn."""
    rc = exf.lib().moe_grouped_product(_p(0), _p(1), _p(2), None, 4, 64, 64, 1, B.EXF_BF16, _p(3), None)
    assert rc == B.EXF_ERR_HIP and B.last_error().startswith("moe_grouped_product:")
