"""Sums that products hold in fp32, for results of every type unless the caller asks for speed, with terms that cancel."""

import pytest

import block8_ref as R
import test_gpu_block8 as B
from block8_shapes import SHAPES

pytestmark = pytest.mark.gpu
hb, torch = B.hb, B.torch


# ---- products -----------------------------------------------------------------------------------------------------------
def check(a, w, y, kind, bias=None, gate=None, add=None, fast=False):
    want, off = R.product(*(R.values64(B.code_bytes(x.codes), x.scales, x.block_rows) for x in (a, w)), bias, gate, add, eight_bit=fast)
    R.check_rounded(y, want, off, B.unit(kind), "product")


def cancelling(rows, cols, block_rows, seed):
    """Codes of small normal deviates but for two neighbouring columns of the first and of the last block, of 256 in activations and of 1 and -1 in weights:
    what eight products around them come to is a ten thousandth of those two."""
    T = torch()
    g = T.Generator(B.DEV).manual_seed(seed)
    x = T.randn((rows, cols), generator=g, device=B.DEV) * (0.5 if block_rows == 1 else 0.1)
    for at in (3, (cols - 1) // 128 * 128):
        x[:, at], x[:, at + 1] = (256.0, 256.0) if block_rows == 1 else (1.0, -1.0)
    held = T.zeros((rows, -(-cols // 16) * 16), dtype=T.uint8, device=B.DEV)
    held[:, :cols] = x.to(T.float8_e4m3fn).view(T.uint8)
    return hb().Block8(held[:, :cols], T.ones((R.blocks_of_rows(rows, block_rows), R.blocks(cols)), device=B.DEV), block_rows)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("gate,m,n,k", [(None, 1, 16, 130), (None, 1, 6144, 1500), (None, 7, 2000, 300), (None, 65, 896, 900), (None, 300, 1024, 500), (None, 4100, 130, 260),
                                        (None, 16640, 1152, 300), ("silu", 1, 8960, 1500), ("silu", 20, 512, 1000), ("gelu", 300, 768, 500), ("silu", 2049, 4096, 130)])
def test_products_whose_terms_cancel(kind, gate, m, n, k):
    """Within the bound of fp32 sums; a row alone is within it too, whichever tile it takes then."""
    a, w = cancelling(m, k, 1, 100 + m), cancelling(n, k, 128, 200 + n)
    check(a, w, hb().block_matmul(a, w, dtype=B.tdt(kind), gate=gate), kind, gate=gate)
    for row in {0, m // 2, m - 1}:
        one = hb().Block8(a.codes[row:row + 1], a.scales[row:row + 1])
        check(one, w, hb().block_matmul(one, w, dtype=B.tdt(kind), gate=gate), kind, gate=gate)


@pytest.mark.parametrize("gated,m,n,k", sorted({s[1:] for s in SHAPES if s[0] == "f32"}))
def test_bf16_products_by_every_shape_of_tile(gated, m, n, k):
    """The sizes at which fp32 results take every shape: bf16 results take the same, with the same sums."""
    for cols, gate in ((k, "silu" if gated else None), (k - k % 128, "gelu" if gated else None)):
        a, w = B.matrix(m, cols, 1, 120), B.matrix(n, cols, 128, 121)
        if gate:
            a.scales.mul_(0.1 / cols ** 0.5)
        check(a, w, hb().block_matmul(a, w, gate=gate), "bf16", gate=gate)
        bias, add = B.draw((n,), 122, "f32", 2.0), B.draw((m, n // 2 if gate else n), 123, "bf16", 2.0)
        check(a, w, hb().block_matmul(a, w, gate=gate, bias=bias, add=add), "bf16", bias, gate, add)


@pytest.mark.parametrize("gated,m,n,k", sorted({s[1:] for s in SHAPES if s[0] == "bf16"}))
def test_bf16_products_of_callers_that_ask_for_speed(gated, m, n, k):
    a, w = B.matrix(m, k, 1, 124), B.matrix(n, k, 128, 125)
    if gated:
        a.scales.mul_(0.1 / k ** 0.5)
    gate, add = "silu" if gated else None, B.draw((m, n // 2 if gated else n), 126, "bf16", 2.0)
    check(a, w, hb().block_matmul(a, w, gate=gate, add=add, fast=True), "bf16", None, gate, add, fast=True)
