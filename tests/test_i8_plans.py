"""The 8-bit product's choice of kernel and pieces of K, as callers rely on it (host only)."""
import random

import pytest

from paper_2505_05286_amd import hxf

from . import i8_instances
from ._lib import ensure_built

EPILOGUES = (hxf.EPI_BF16, hxf.EPI_RESID, hxf.EPI_SWIGLU, hxf.EPI_F32)


@pytest.fixture(autouse=True)
def _built():
    ensure_built()


def _partials(m, n, k):
    """Bytes that the pieces of the product's plan take, of the epilogue that takes most."""
    pieces = [hxf.op_gemm_i8_plan(m, n, k, e)[4] for e in EPILOGUES if e != hxf.EPI_SWIGLU or n % 2 == 0]
    return max((p * m * n * 4 if p > 1 else 0) for p in pieces)


# projections of 4096, 5120 and 8192 wide layers (columns as the call counts them), and an odd one
@pytest.mark.parametrize("n,k", [(6144, 4096), (4096, 4096), (28672, 4096), (4096, 14336), (7168, 5120), (55296, 5120),
                                 (5120, 27648), (10240, 8192), (57344, 8192), (8192, 28672), (777, 28672)])
def test_the_workspace_of_the_largest_batch_serves_all_smaller_ones(n, k):
    rows = [*range(1, 700), *range(700, 2081, 23), 2080]
    most = 0
    for m in rows:
        most = max(most, _partials(m, n, k))
        assert most <= hxf.op_gemm_i8_workspace_bytes(m, n, k) <= hxf.GEMM_I8_MAX_WORKSPACE, m


def test_the_workspace_covers_smaller_products_of_any_size():
    r = random.Random(3)

    def size(lo, hi):
        return int(round(2 ** r.uniform(lo, hi)))
    cut = 0
    for _ in range(30000):
        m, n, k = size(0, 12), size(0, 17), size(6, 17 - 1e-5)
        need = _partials(m, n, k)
        cut += need > 0
        assert need <= hxf.op_gemm_i8_workspace_bytes(m, n, k)
        assert need <= hxf.op_gemm_i8_workspace_bytes(m + size(0, 12), n + size(0, 15), min(k + size(0, 16), (1 << 17) - 1))
    assert cut > 1000
    assert hxf.op_gemm_i8_workspace_bytes(100000, 100000, 131071) == hxf.GEMM_I8_MAX_WORKSPACE
    assert hxf.op_gemm_i8_workspace_bytes(0, 4096, 14336) == 0


def test_every_compiled_instance_is_taken_by_a_tested_product():
    """With its epilogue: the instances are compiled for each of them."""
    taken = {i8_instances.instance(*p) for p in i8_instances.products()}
    every = i8_instances.compiled()
    assert len(every) == 41 * 6 + 6 * 4
    assert taken == every, (sorted(every - taken), sorted(taken - every))
