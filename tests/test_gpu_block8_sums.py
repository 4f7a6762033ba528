"""Sums that products and norms hold in fp32: products into every type unless the caller asks for speed, with terms that cancel; heads whose squares are below
fp32's range."""

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


# ---- norms --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("channels", [1, 7, 128, 200, 250, 300, 520, 1000, 1030, 2056, 4096, 4104, 8200, 12000, 16392, 20000])
def test_norm_of_heads_whose_squares_are_below_fp32(kind, channels):
    """Heads of every size down to fp32's least beside each other and beside zeros.  A square's rounding is 2^-150 at most where it is below fp32's normal range,
    which matters up to 2^-120: a root of 2^-30 more, relative to it, beyond what larger heads may be off."""
    T = torch()
    sizes = [1e-19, 1.0, 1e-23, 0.0, 1e-30, 3e-38, 1e-17, 1e-41, 1e-18, 1e-21, 1e4]
    x = B.draw((len(sizes), channels), 130, "f32").cpu().double() * T.tensor(sizes, dtype=T.float64)[:, None]
    x = x.float().to(B.tdt(kind)).to(B.DEV)
    gain = B.draw((channels,), 131).abs() + 0.5
    for eps in (0.0, 1e-42, 2.0 ** -125, 2.0 ** -119, 1e-30):
        held = float(T.tensor(eps, dtype=T.float32))
        out, total, q = hb().rms_norm(x, gain, eps=eps, total=True, block8=True)
        assert T.equal(total, x)
        _, y = R.norm(B.to64(x), None, B.to64(gain), held, 0.0)
        off = (R.norm_slack(channels) + 2 * R.U32 + 2.0 ** -30) * abs(y)
        # y below its type's normal range would be off by half of the least value: of s / size in fp32, times gains below 8, and of bf16
        R.check_rounded(B.to64(out), y, off + 2.0 ** -146 + (2.0 ** -134 if kind == "bf16" else 0.0), B.unit(kind), f"eps {eps}")
        R.check_codes(B.code_bytes(q.codes).cpu(), B.to64(q.scales), y, off + 2.0 ** -146, f"eps {eps}")
        again = hb().rms_norm(x, gain, eps=eps, out=x.clone())[0]
        assert T.equal(again, out)


@pytest.mark.parametrize("heads,channels", [(5, 64), (32, 128), (3, 200), (2, 1000), (3, 1500)])
def test_norm_of_small_heads_beside_large_ones(heads, channels):
    """Heads of one token of both kinds, so that lanes of one wavefront and workgroup differ."""
    T = torch()
    x = B.draw((37, heads, channels), 132)
    x[::3, ::2] *= 1e-25
    x[1::4, 1::2] = 0.0
    out, _, _ = hb().rms_norm(x, eps=0.0)
    _, y = R.norm(B.to64(x), None, None, 0.0, 0.0)
    R.check_rounded(B.to64(out), y, (R.norm_slack(channels) + 2 * R.U32 + 2.0 ** -30) * abs(y), R.U32)
