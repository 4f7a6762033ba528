"""Products by every way through the kernels' loop over k, with columns that end inside 16 (block8_edges.py)."""

import pytest

import block8_ref as R
import test_gpu_block8 as B
from block8_edges import EDGES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,gated,m,n,k", EDGES)
def test_product_by_every_way_through_the_loop(kind, gated, m, n, k):
    gate, fast = "silu" if gated else None, kind.endswith("fast")
    B.run_and_check(kind, m, n, k, gate, 140)
    if kind.startswith("f32"):                                           # bf16 results take the same tiles
        a, w = B.matrix(m, k, 1, 142), B.matrix(n, k, 128, 143)
        if gate:
            a.scales.mul_(0.1 / k ** 0.5)
        add = B.draw((m, n // 2 if gate else n), 144, "bf16", 2.0)
        want, off = R.product(*(R.values64(B.code_bytes(x.codes), x.scales, x.block_rows) for x in (a, w)), None, gate, add, eight_bit=fast)
        R.check_rounded(B.hb().block_matmul(a, w, gate=gate, add=add, fast=fast), want, off, R.UBF, "product")
