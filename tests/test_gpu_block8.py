"""The operators of a layer's projections in 8 bits, through the Python entry points, against 64-bit references (block8_ref.py) with bounds
derived there."""

import numpy as np
import pytest

import block8_ref as R
from block8_shapes import SHAPES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def hb():
    from paper_2504_02921_amd import binding
    return binding


def torch():
    import torch
    return torch


def tdt(kind):
    return torch().float32 if kind.startswith("f32") else torch().bfloat16


def unit(kind):
    return R.U32 if kind.startswith("f32") else R.UBF


def to64(t):
    return t.detach().double().cpu().numpy()


def code_bytes(t):
    return t.contiguous().view(torch().uint8)


def gen(seed):
    return torch().Generator().manual_seed(seed)


def draw(shape, seed, kind="f32", size=1.0):
    return (torch().randn(shape, generator=gen(seed)) * size).to(tdt(kind)).to(DEV)


# ---- norm ---------------------------------------------------------------------------------------------------------------
def check_norm(x, gain, add, eps, offset, out, total, block8, kind):
    s, y = R.norm(to64(x), None if add is None else to64(add), None if gain is None else to64(gain), eps, offset)
    g = 1.0 if gain is None else np.abs(to64(gain)) + abs(offset)
    off = R.norm_slack(x.shape[-1]) * np.abs(y) + 2 * R.U32 * np.abs(y) + (0.0 if gain is None else R.U32 * np.abs(y) / np.maximum(np.abs(to64(gain) + offset), 1e-30) * g)
    if total is not None:
        R.check_rounded(to64(total), s, R.U32 * np.abs(s), unit(kind) if kind == "bf16" else 0.0, "total")
    if out is not None:
        R.check_rounded(to64(out), y, off, unit(kind), "out")
    if block8 is not None:
        R.check_codes(code_bytes(block8.codes).cpu(), to64(block8.scales), y, off, "codes")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,channels", [(1, 1), (3, 2), (5, 7), (1, 128), (7, 129), (33, 100), (2, 256), (9, 250), (4, 512), (65, 896), (6, 1000), (3, 2048), (1030, 2500),
                                             (1024, 512), (1500, 127), (1025, 4096), (5, 4864), (2, 16384), (3, 16385), (2, 40001)])
def test_norm_is_the_formula(kind, tokens, channels):
    x, add, gain = draw((tokens, channels), 1, kind, 3.0), draw((tokens, channels), 2, kind), draw((channels,), 3)
    out, total, q = hb().rms_norm(x, gain, add=add, eps=1e-5, gain_offset=1.0, total=True, block8=True)
    check_norm(x, gain, add, 1e-5, 1.0, out, total, q, kind)
    out, total, q = hb().rms_norm(x)
    assert total is None and q is None
    check_norm(x, None, None, 1e-6, 0.0, out, None, None, kind)
    out, total, q = hb().rms_norm(x, gain, out=False, block8=True)
    assert out is None and total is None
    check_norm(x, gain, None, 1e-6, 0.0, None, None, q, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("channels", [120, 136, 250, 264, 504, 520, 1016, 1032, 2040, 2056, 4095, 4104, 8191, 8200, 16383, 16392])
def test_norm_by_every_number_of_lanes(kind, channels):
    """On both sides of each number of channels behind which more lanes, more chunks or a second reading take over, with few rows and many."""
    for tokens in (3, 255, 257):
        x, add, gain = draw((tokens, channels), 21, kind, 3.0), draw((tokens, channels), 22, kind), draw((channels,), 23)
        check_norm(x, gain, add, 1e-5, 0.0, *hb().rms_norm(x, gain, add=add, eps=1e-5, total=True, block8=True), kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,heads,channels", [(1, 1, 64), (5, 14, 64), (3, 32, 128), (2, 5, 80), (7, 3, 96), (4, 2, 256), (1, 2, 300), (50, 32, 600)])
def test_norm_of_heads_in_rows_of_a_projection(kind, tokens, heads, channels):
    rows = draw((tokens, (heads + 2) * channels + 3), 4, kind)
    x = rows[:, 1:1 + heads * channels].unflatten(1, (heads, channels))
    gain = draw((channels,), 5)
    out, _, _ = hb().rms_norm(x, gain)
    check_norm(x, gain, None, 1e-6, 0.0, out, None, None, kind)
    before = rows.clone()
    hb().rms_norm(x, gain, out=x)                                       # in place, the other columns untouched
    assert torch().equal(x, out)
    x.copy_(before[:, 1:1 + heads * channels].unflatten(1, (heads, channels)))
    assert torch().equal(rows, before)
    by_channel = draw((heads, tokens, channels), 6, kind).transpose(0, 1)
    check_norm(by_channel, gain, None, 1e-6, 0.0, hb().rms_norm(by_channel, gain)[0], None, None, kind)


@pytest.mark.parametrize("channels", [96, 2000, 4096, 20000])
def test_norm_in_place_and_onto_the_stream(channels):
    T = torch()
    for tokens in (3, 1100):
        x, add, gain = draw((tokens, channels), 7, "bf16"), draw((tokens, channels), 8, "bf16"), draw((channels,), 9)
        out, total, _ = hb().rms_norm(x, gain, add=add, total=True)
        xs, ad = x.clone(), add.clone()
        o, t, _ = hb().rms_norm(xs, gain, add=ad, out=ad, total=xs)
        assert o is ad and t is xs and T.equal(xs, total) and T.equal(ad, out)
        xs, ad = x.clone(), add.clone()
        o, t, _ = hb().rms_norm(xs, gain, add=ad, out=xs, total=ad)
        assert T.equal(ad, total) and T.equal(xs, out)


def test_norm_of_zeros_and_of_what_is_not_finite():
    T = torch()
    x = T.zeros((6, 300), device=DEV)
    x[1, 5], x[2, 299], x[3, 0] = float("nan"), float("inf"), 1e30
    x[4] = 1e-30
    for eps in (0.0, 1e-6):
        out, _, q = hb().rms_norm(x, eps=eps, block8=True)
        assert not out[0].any() and not q.codes[0].float().any() and (q.scales[0] == 1).all() and (q.scales[5] == 1).all()
        assert out[1].isnan().all() and q.codes[1].float().isnan().all() and (q.scales[1] == 1).all()       # as the sum is
        assert out[2, 299].isnan() and not out[2, :299].any()                                               # 1 / infinity, and infinity / infinity
        assert not out[3].any()                                                                             # squares past fp32
        assert not out[5].any()
    assert (hb().rms_norm(x, eps=1e-6)[0][4] > 0).all()


def test_norm_takes_no_tokens_and_views():
    T = torch()
    out, total, q = hb().rms_norm(T.empty((0, 64), device=DEV), total=True, block8=True)
    assert out.shape == (0, 64) and total.shape == (0, 64) and q.shape == (0, 64)
    wide = draw((9, 1000), 10)
    x = wide[::2, 3:700]
    y = T.full((9, 1000), 7.0, device=DEV)
    held = hb().Block8(T.full((5, 704), 0x55, dtype=T.uint8, device=DEV)[:, :697], T.empty((5, 6), device=DEV))
    out, _, q = hb().rms_norm(x, out=y[::2, 3:700], block8=held)
    assert q is held and out.data_ptr() == y[::2, 3:700].data_ptr()
    check_norm(x, None, None, 1e-6, 0.0, out, None, q, "f32")
    assert (y[1::2] == 7).all() and (y[:, :3] == 7).all() and (y[:, 700:] == 7).all()
    one = T.as_strided(held.codes, (5, 704), (704, 1))
    assert (one[:, 697:] == 0x55).all()                                  # a row's padding is not written
    row = draw((1, 200), 11).expand(4, 200)                              # the same row for all
    assert T.equal(hb().rms_norm(row)[0], hb().rms_norm(row.contiguous())[0])


# ---- codes --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 100), (127, 129), (128, 128), (129, 257), (300, 1000), (17, 5), (260, 4864)])
def test_codes_are_the_definitions(kind, block_rows, rows, cols):
    x = draw((rows, cols), 12, kind)
    x = x * torch().exp(draw((1, cols), 13, kind) * 2)
    x[rows // 2] *= 1e-3
    q = hb().block_quantize(x, block_rows=block_rows)
    codes, scales = R.quantize(x.float().cpu().numpy(), block_rows)
    np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
    got = code_bytes(q.codes).cpu().numpy()
    np.testing.assert_array_equal(np.where(got == 0x80, 0, got), np.where(codes == 0x80, 0, codes))


def test_codes_of_every_size_and_of_what_is_not_finite():
    T = torch()
    x = T.zeros((140, 300))
    x[0] = T.linspace(-5.0, 5.0, 300)
    x[1] = 1e-40 * T.linspace(-5.0, 5.0, 300)                           # below the least scale
    x[2] = 3e38 * T.linspace(-1.0, 1.0, 300)
    x[3, 7], x[3, 8], x[3, 9], x[3, 10] = float("nan"), float("inf"), -float("inf"), 2.0
    x[4, 150] = float("inf")
    x[139, 299] = -7.0
    for block_rows in (1, 128):
        for cols in (300, 299):
            y = x[:, :cols].contiguous().to(DEV)
            q = hb().block_quantize(y, block_rows=block_rows)
            codes, scales = R.quantize(y.cpu().numpy(), block_rows)
            np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
            got, want = q.codes.float().cpu().numpy(), R.ofp8.e4m3_decode(codes)
            np.testing.assert_array_equal(got, want)                    # NaN equals NaN here
            assert np.isnan(got[3, 7:10]).all() and np.isnan(got[4, 150])


def test_codes_into_a_matrix_in_hand_and_of_views():
    T = torch()
    wide = draw((300, 1000), 14, "bf16")
    for block_rows in (1, 128):
        x = wide[1::2, 5:405]
        codes = T.full((150, 512), 0x33, dtype=T.uint8, device=DEV)
        held = hb().Block8(codes[:, :400], T.full((150 if block_rows == 1 else 2, 9), -1.0, device=DEV)[:, 2:6], block_rows)
        q = hb().block_quantize(x, block_rows=block_rows, out=held)
        assert q is held and (codes[:, 400:] == 0x33).all()
        want = hb().block_quantize(x.contiguous(), block_rows=block_rows)
        assert T.equal(held.codes, want.codes.view(T.uint8)) and T.equal(held.scales, want.scales)


# ---- product ------------------------------------------------------------------------------------------------------------
def matrix(rows, cols, block_rows, seed, pad=0x7F):
    """Codes of normal deviates under scales of many sizes, in rows whose padding holds codes that are NaN."""
    T = torch()
    g = T.Generator(DEV).manual_seed(1000 * seed + rows + cols)
    held = T.full((rows, R.blocks(cols) * 128 + 16), pad, dtype=T.uint8, device=DEV)
    held[:, :cols] = (T.randn((rows, cols), generator=g, device=DEV) * 60.0).to(T.float8_e4m3fn).view(T.uint8)
    return hb().Block8(held[:, :cols], T.randn((R.blocks_of_rows(rows, block_rows), R.blocks(cols)), generator=g, device=DEV).exp(), block_rows)


def check_product(a, w, y, kind, bias=None, gate=None, add=None):
    want, off = R.product(*(R.values64(x.codes.view(torch().uint8), x.scales, x.block_rows) for x in (a, w)), bias, gate, add, eight_bit=kind == "bf16" or kind.endswith("fast"))
    if kind.startswith("block8"):
        R.check_codes(code_bytes(y.codes), y.scales, want, off, "product")
    else:
        R.check_rounded(y, want, off, unit(kind), "product")


def run_and_check(kind, m, n, k, gate=None, seed=20):
    """Without and with what may follow the product."""
    a, w = matrix(m, k, 1, seed), matrix(n, k, 128, seed + 1)
    if gate:
        a.scales.mul_(0.1 / k ** 0.5)                                    # a gate's interesting arguments
    wide, fast = n // 2 if gate else n, kind.endswith("fast")
    bias = draw((n,), 22, "f32", 2.0 if gate else 100.0)
    if kind.startswith("block8"):
        check_product(a, w, hb().block_matmul(a, w, gate=gate, block8=True, fast=fast), kind, None, gate)
        return check_product(a, w, hb().block_matmul(a, w, gate=gate, bias=bias, block8=True, fast=fast), kind, bias, gate)
    check_product(a, w, hb().block_matmul(a, w, dtype=tdt(kind), gate=gate, fast=fast), kind, None, gate)
    add = draw((m, wide), 23, kind, 2.0 if gate else 100.0)
    check_product(a, w, hb().block_matmul(a, w, gate=gate, bias=bias, add=add, fast=fast), kind, bias, gate, add)


@pytest.mark.parametrize("kind", ["bf16", "f32", "block8"])
@pytest.mark.parametrize("m,n,k", [(1, 16, 32), (1, 1, 1), (2, 3, 5), (1, 200, 128), (16, 32, 256), (17, 33, 129), (5, 130, 1000), (33, 96, 300), (64, 128, 130), (65, 100, 896),
                                   (70, 257, 2500), (130, 300, 640), (129, 128, 127), (300, 384, 400), (257, 513, 384), (200, 64, 4864), (1, 640, 4100), (700, 1000, 1030)])
def test_product_is_the_sum_over_blocks(kind, m, n, k):
    run_and_check(kind, m, n, k)


@pytest.mark.parametrize("kind", ["bf16", "f32", "block8"])
@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("m,n,k", [(1, 256, 128), (3, 512, 100), (20, 256, 1000), (40, 768, 256), (65, 512, 640), (140, 256, 300), (300, 768, 500)])
def test_gated_product(kind, gate, m, n, k):
    run_and_check(kind, m, n, k, gate)


@pytest.mark.parametrize("kind,gated,m,n,k", SHAPES)
def test_product_of_every_shape_of_tile(kind, gated, m, n, k):
    run_and_check(kind, m, n, k, "silu" if gated else None)
    run_and_check(kind, m, n, k - k % 128, "gelu" if gated else None, 25)


@pytest.mark.parametrize("m", [3, 40, 300])
def test_product_onto_the_stream_and_into_views(m):
    T = torch()
    a, w = matrix(m, 500, 1, 28), matrix(200, 500, 128, 29)
    stream = draw((2 * m, 211), 30, "bf16", 50.0)
    before, x = stream.clone(), stream[::2, 3:203]
    y = hb().block_matmul(a, w, add=x)
    check_product(a, w, y, "bf16", None, None, before[::2, 3:203])
    assert hb().block_matmul(a, w, add=x, out=x) is x and T.equal(x, y)
    stream[::2, 3:203] = before[::2, 3:203]
    assert T.equal(stream, before)                                       # nothing but those rows and columns


@pytest.mark.parametrize("kind", ["bf16", "f32", "block8"])
def test_a_code_that_is_nan_stays_in_its_row_or_column(kind):
    T = torch()
    for m in (5, 200):
        a, w = matrix(m, 300, 1, 31), matrix(384, 300, 128, 32)
        run = (lambda: hb().block_matmul(a, w, block8=True).codes.float()) if kind == "block8" else (lambda: hb().block_matmul(a, w, dtype=tdt(kind)).float())
        clean = run()
        assert not clean.isnan().any()
        a.codes[m - 2, 299] = 0x7F
        got = run()
        keep = T.arange(m, device=DEV) != m - 2
        assert got[m - 2].isnan().all() and T.equal(got[keep], clean[keep])
        w.codes[7, 3] = 0xFF
        got = run()
        keep_n = T.arange(384, device=DEV) != 7
        assert got[:, 7].isnan().all() and T.equal(got[keep][:, 128:], clean[keep][:, 128:])
        if kind != "block8":                                             # its block's scale may be another one
            assert T.equal(got[keep][:, keep_n], clean[keep][:, keep_n])


def test_product_of_nothing():
    T, H = torch(), hb()
    a, w = matrix(4, 64, 1, 33), matrix(256, 64, 128, 34)
    empty_a, empty_w = H.Block8.empty(0, 64), H.Block8.empty(0, 64, 128)
    assert H.block_matmul(empty_a, w).shape == (0, 256) and H.block_matmul(a, empty_w).shape == (4, 0)
    assert H.block_matmul(empty_a, w, gate="silu", block8=True).shape == (0, 128)
    assert H.block_quantize(T.empty((0, 64), device=DEV)).shape == (0, 64)


def test_the_same_bits_again_and_on_other_streams():
    T, H = torch(), hb()
    x, add, gain = draw((300, 900), 35, "bf16"), draw((300, 900), 36, "bf16"), draw((900,), 37)
    up, down = H.block_quantize(draw((512, 900), 38), 128), H.block_quantize(draw((900, 256), 39), 128)

    def layer(stream=None):
        _, total, q = H.rms_norm(x, gain, add=add, out=None, total=True, block8=True, stream=stream)
        h = H.block_matmul(q, up, gate="silu", block8=True, stream=stream)
        return total, q.codes, h.codes, h.scales, H.block_matmul(h, down, add=total, stream=stream)

    first = layer()
    T.cuda.synchronize()
    side = T.cuda.Stream()
    for stream in (None, side, side):
        side.wait_stream(T.cuda.current_stream())
        got = layer(stream)
        T.cuda.synchronize()
        assert all(T.equal(a.view(T.uint8) if a.dtype == T.float8_e4m3fn else a, b.view(T.uint8) if b.dtype == T.float8_e4m3fn else b) for a, b in zip(first, got))


@pytest.mark.parametrize("m", [1, 20, 300])
def test_a_feed_forward_layer_step_by_step_and_recorded(m):
    """norm -> gated product -> product onto the stream -> norm, each step against the reference on what the steps before it gave; then the same recorded
    into a graph and replayed on other values."""
    T, H = torch(), hb()
    hidden, ffn = 500, 384
    gain = draw((hidden,), 40)
    w_up, w_down = draw((2 * ffn, hidden), 41, "bf16", 0.05), draw((hidden, ffn), 42, "bf16", 0.05)
    up, down = H.block_quantize(w_up, 128), H.block_quantize(w_down, 128)
    x, add = draw((m, hidden), 43, "bf16"), draw((m, hidden), 44, "bf16")
    q, h = H.Block8.empty(m, hidden), H.Block8.empty(m, ffn)
    total, out, last = T.empty_like(x), T.empty_like(x), T.empty_like(x)

    def layer():
        H.rms_norm(x, gain, add=add, out=None, total=total, block8=q)
        H.block_matmul(q, up, gate="silu", block8=h)
        H.block_matmul(h, down, add=total, out=out)
        H.rms_norm(out, gain, out=last)

    layer()
    check_norm(x, gain, add, 1e-6, 0.0, None, total, q, "bf16")
    check_product(q, up, h, "block8", None, "silu")
    check_product(h, down, out, "bf16", None, None, total)
    check_norm(out, gain, None, 1e-6, 0.0, last, None, None, "bf16")
    graph = T.cuda.CUDAGraph()
    side = T.cuda.Stream()
    side.wait_stream(T.cuda.current_stream())
    with T.cuda.stream(side):
        layer()
    T.cuda.current_stream().wait_stream(side)
    with T.cuda.graph(graph):
        layer()
    for seed in range(3):
        x.copy_(draw((m, hidden), 50 + seed, "bf16"))
        layer()
        want = [t.clone() for t in (total, out, last, h.scales)]
        for t in (total, out, last, h.scales):
            t.zero_()
        graph.replay()
        T.cuda.synchronize()
        assert all(T.equal(a, b) for a, b in zip(want, (total, out, last, h.scales)))


# ---- places far apart ---------------------------------------------------------------------------------------------------
def same(a, b):
    if isinstance(a, hb().Block8):
        return torch().equal(code_bytes(a.codes), code_bytes(b.codes)) and torch().equal(a.scales, b.scales)
    return torch().equal(a, b)


def apart(rows, cols, block_rows=1, like=None, stride=1 << 22):
    """A matrix whose rows are `stride` bytes apart, with the codes of `like`."""
    T = torch()
    codes = T.empty((rows - 1) * stride + R.blocks(cols) * 128, dtype=T.uint8, device=DEV).as_strided((rows, cols), (stride, 1))
    if like is not None:
        codes.copy_(code_bytes(like.codes))
    scales = T.empty((R.blocks_of_rows(rows, block_rows), R.blocks(cols)), device=DEV) if like is None else like.scales
    return hb().Block8(codes, scales, block_rows)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_heads_past_four_gib(kind):
    T = torch()
    place = lambda: T.empty((1 << 32) + (1 << 30) + 300, dtype=tdt(kind), device=DEV).as_strided((3, 2, 300), (1 << 31, 1 << 30, 1))      # noqa: E731
    x, add, gain = draw((3, 2, 300), 70, kind), draw((3, 2, 300), 71, kind), draw((300,), 72)
    far = [place() for _ in range(3)]
    far[0].copy_(x)
    out, total, _ = hb().rms_norm(x, gain, add=add, total=True)
    hb().rms_norm(far[0], gain, add=add, total=far[1], out=far[2])
    assert T.equal(far[1], total) and T.equal(far[2], out)


def test_codes_past_four_gib():
    x = draw((1100, 300), 73)
    q = apart(1100, 300)
    assert same(hb().rms_norm(x, out=None, block8=q)[2], hb().rms_norm(x, out=None, block8=True)[2])
    assert same(hb().block_quantize(x, out=q), hb().block_quantize(x))
    q = apart(1100, 300, 128)
    assert same(hb().block_quantize(x, 128, out=q), hb().block_quantize(x, 128))
    rows = torch().empty((1099 << 21) + 300, device=DEV).as_strided((1100, 300), (1 << 21, 1))
    rows.copy_(x)
    assert same(hb().block_quantize(rows), hb().block_quantize(x))


@pytest.mark.parametrize("kind", ["bf16", "f32", "block8"])
@pytest.mark.parametrize("m,n,stride", [(20, 1152, 1 << 22), (1100, 1152, 1 << 22), (16640, 4096, 1 << 19)])
def test_products_past_four_gib(kind, m, n, stride):
    T, k = torch(), 300
    a, w = matrix(m, k, 1, 74), matrix(n, k, 128, 75)
    fa, fw = apart(m, k, 1, a, stride if m > 1000 else 1 << 22), apart(n, k, 128, w)
    if kind == "block8":
        assert same(hb().block_matmul(fa, fw, block8=apart(m, n, stride=stride)), hb().block_matmul(a, w, block8=True))
        return
    out = T.empty((m - 1) * (stride >> 1) + n, dtype=tdt(kind), device=DEV).as_strided((m, n), (stride >> 1, 1))
    add = draw((m, n), 76, kind)
    assert same(hb().block_matmul(fa, fw, add=add, out=out), hb().block_matmul(a, w, add=add))


def test_more_rows_than_a_launch_has_workgroups():
    """1 100 000 rows, a thousand over and over: workgroups walk rows, and every row is the same as alone."""
    T, n, times = torch(), 1000, 1100
    few = draw((n, 2056), 77, "bf16")
    x = few.repeat(times, 1)
    gain = draw((2056,), 78)
    out, _, q = hb().rms_norm(x, gain, block8=True)
    want, _, wq = hb().rms_norm(few, gain, block8=True)
    whole = lambda t: t.view(times, n, -1)                               # noqa: E731
    assert (whole(out) == want).all()
    assert (whole(code_bytes(q.codes)) == code_bytes(wq.codes)).all() and (whole(q.scales) == wq.scales).all()
    del out
    q, wq = hb().block_quantize(x, out=q), hb().block_quantize(few)
    assert (whole(code_bytes(q.codes)) == code_bytes(wq.codes)).all() and (whole(q.scales) == wq.scales).all()
    w = matrix(100, 2056, 128, 79)
    y = hb().block_matmul(q, w)
    for at in (0, 777, times - 1):
        check_product(wq, w, y[at * n:(at + 1) * n], "bf16")


# ---- several at once ----------------------------------------------------------------------------------------------------
def test_layers_from_two_threads_on_streams_of_their_own():
    """Nothing is kept between calls, so calls of several host threads at once give the bits of the same calls alone."""
    import threading
    T, H = torch(), hb()
    up, down = H.block_quantize(draw((512, 700), 80), 128), H.block_quantize(draw((700, 256), 81), 128)
    xs = [draw((m, 700), 82 + m, "bf16") for m in (3, 290)]

    def layer(x):
        _, total, q = H.rms_norm(x, out=None, total=True, block8=True)
        return H.block_matmul(H.block_matmul(q, up, gate="gelu", block8=True), down, add=total)

    want = [layer(x) for x in xs]
    T.cuda.synchronize()
    got = [[], []]

    def work(i):
        with T.cuda.stream(T.cuda.Stream()):
            got[i] = [layer(xs[i]) for _ in range(20)]
            T.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert all(len(g) == 20 and all(T.equal(y, want[i]) for y in g) for i, g in enumerate(got))


def test_matrices_that_are_let_go_stay_until_their_stream_is_done():
    """A call on another stream keeps what it reads: memory that the caller lets go while it waits there is not given to anybody else."""
    T, H = torch(), hb()
    x, up, busy = draw((300, 900), 90, "bf16"), H.block_quantize(draw((512, 900), 91), 128), T.randn((4096, 4096), device=DEV)
    want = H.block_matmul(H.block_quantize(x), up)
    T.cuda.synchronize()
    side = T.cuda.Stream()
    with T.cuda.stream(side):
        for _ in range(20):
            T.mm(busy, busy)
    side.wait_stream(T.cuda.current_stream())
    held = x.clone()
    q = H.block_quantize(held)
    side.wait_stream(T.cuda.current_stream())
    total = H.rms_norm(held, out=False, total=True, stream=side)[1]
    y = H.block_matmul(q, up, stream=side)
    places = {held.data_ptr(), q.codes.data_ptr()}
    del held, q
    fresh = [T.zeros_like(x), H.Block8.empty(300, 900)]
    assert not places & {fresh[0].data_ptr(), fresh[1].codes.data_ptr()}
    T.cuda.synchronize()
    assert T.equal(total, x) and T.equal(y, want)


def test_two_branches_of_one_recording():
    """Two products on two streams of one recording, each with a second launch for its last rows, replayed on other values."""
    T, H = torch(), hb()
    m, n, k = 16640, 4096, 300
    a, w = matrix(m, k, 1, 84), [matrix(n, k, 128, s) for s in (85, 86)]
    outs = [T.empty((m, n), dtype=T.bfloat16, device=DEV) for _ in w]
    for i in range(2):
        H.block_matmul(a, w[i], out=outs[i])
    T.cuda.synchronize()
    graph, side = T.cuda.CUDAGraph(), T.cuda.Stream()
    with T.cuda.graph(graph):
        side.wait_stream(T.cuda.current_stream())
        H.block_matmul(a, w[0], out=outs[0])
        with T.cuda.stream(side):
            H.block_matmul(a, w[1], out=outs[1])
        T.cuda.current_stream().wait_stream(side)
    for seed in (87, 88):
        fresh = matrix(m, k, 1, seed)
        a.codes.copy_(fresh.codes)
        a.scales.copy_(fresh.scales)
        want = [H.block_matmul(fresh, x) for x in w]
        [o.zero_() for o in outs]
        graph.replay()
        T.cuda.synchronize()
        assert all(T.equal(x, y) for x, y in zip(want, outs))


def test_the_demos_layer_runs():
    """Norms, projections, rotary positions and attention in one layer, over a pool with documents of several lengths.  Rounding both operands of a
    product to E4M3 moves it by 2^-5 of itself or so (half a step of 2^-4, uniform over it: 2^-4 / 3^0.5 each at most); the gated branch multiplies two such."""
    from paper_2504_02921_amd import demo, workloads
    import numpy
    T, cfg, rng = torch(), workloads.ModelCfg("layer", 1, 256, 4, 2, 64, 384, 500, 1e6, 1e-6, dtype="bf16"), numpy.random.default_rng(3)
    docs = [rng.integers(0, cfg.vocab, n).astype(numpy.int32) for n in (40, 130)]
    pool = hb().KVPool(1, cfg.n_kv_heads, cfg.head_dim, 16, "bf16", DEV)
    model = hb().Model(cfg, workloads.SeededWeights(cfg, seed=1, std=0.05), DEV)
    try:
        pages = [pool.alloc(-(-len(d) // hb().PAGE_TOKENS)) for d in docs]
        model.doc_prefill(pool, docs, pages)
        gap, away = demo.layer_of_the_callers(pool, cfg, docs, pages, [5, 9])
        T.cuda.synchronize()
        assert numpy.isfinite(gap) and 0 < away < 0.25
    finally:
        model.close()
        pool.close()


# ---- refusals of the binding --------------------------------------------------------------------------------------------
def test_wrong_tensors_are_refused():
    T, H = torch(), hb()
    x = draw((4, 64), 60, "bf16")

    def refused(call, status=None):
        with pytest.raises(H.HrError) as e:
            call()
        assert status is None or e.value.status == status

    refused(lambda: H.rms_norm(x.half()))
    refused(lambda: H.rms_norm(x, x))                                                     # gains are fp32
    refused(lambda: H.rms_norm(x, add=x.float()))
    refused(lambda: H.rms_norm(x, add=x[:3]))
    refused(lambda: H.rms_norm(x.t()))
    refused(lambda: H.rms_norm(x, out=False))
    refused(lambda: H.rms_norm(x, total=x, out=x))
    refused(lambda: H.rms_norm(x, out=x[:1].expand(4, 64)))
    refused(lambda: H.rms_norm(x.unflatten(1, (2, 32)), block8=True))
    refused(lambda: H.rms_norm(x, block8=H.Block8.empty(4, 65)))
    refused(lambda: H.rms_norm(x, eps=-1.0))
    refused(lambda: H.rms_norm(x.cpu()))
    refused(lambda: H.rms_norm(x.float().requires_grad_()))
    refused(lambda: H.rms_norm(x, draw((64,), 61).requires_grad_()))
    refused(lambda: H.block_quantize(x, block_rows=64))
    refused(lambda: H.block_quantize(x[0]))
    refused(lambda: H.block_quantize(x, out=H.Block8.empty(4, 64, 128)))
    refused(lambda: H.Block8(T.empty((4, 100), dtype=T.uint8, device=DEV), T.empty((4, 1), device=DEV)))      # rows 100 bytes apart
    refused(lambda: H.Block8(T.empty((4, 128), dtype=T.uint8, device=DEV)[:, 8:], T.empty((4, 1), device=DEV)))
    refused(lambda: H.Block8(T.empty((4, 128), dtype=T.uint8, device=DEV), T.empty((4, 2), device=DEV)))
    refused(lambda: H.Block8(T.empty((4, 128), dtype=T.int8, device=DEV), T.empty((4, 1), device=DEV)))
    a, w = H.block_quantize(x), H.block_quantize(draw((256, 64), 62), 128)
    refused(lambda: H.block_matmul(w, w))
    refused(lambda: H.block_matmul(a, a))
    refused(lambda: H.block_matmul(a, H.block_quantize(draw((256, 65), 63), 128)), H.HR_ERR_MISMATCH)
    refused(lambda: H.block_matmul(a, H.block_quantize(draw((128, 64), 64), 128), gate="silu"), H.HR_ERR_MISMATCH)
    refused(lambda: H.block_matmul(a, w, gate="relu"))
    refused(lambda: H.block_matmul(a, w, dtype=T.float16))
    refused(lambda: H.block_matmul(a, w, dtype=T.float32, out=T.empty((4, 256), dtype=T.bfloat16, device=DEV)))
    refused(lambda: H.block_matmul(a, w, add=T.empty((4, 128), device=DEV)))
    refused(lambda: H.block_matmul(a, w, bias=T.empty(128, device=DEV)))
    refused(lambda: H.block_matmul(a, w, add=x, block8=True))
    refused(lambda: H.block_matmul(a, w, block8=H.Block8.empty(4, 128)))
    refused(lambda: H.block_matmul(a, w, bias=T.zeros(256, device=DEV).requires_grad_()))
    refused(lambda: H.block_matmul(H.Block8(a.codes, a.scales.clone().requires_grad_()), w))
    with T.no_grad():
        H.rms_norm(x.float().requires_grad_(), draw((64,), 61).requires_grad_())
