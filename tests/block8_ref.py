"""64-bit references of the operators of a layer's projections in 8 bits (the norm with the residual's addition, codes with scales, products of such
matrices), and bounds on what rounding may add."""

import numpy as np

from oracle import fp8 as ofp8

BLOCK = 128
U32, UBF, U8 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -4      # half a step of fp32, bf16, E4M3 relative to the value
TOP = 448.0


def blocks(n):
    return -(-n // BLOCK)


def spread(scales, rows, cols, block_rows):
    """The scale of every value."""
    return np.repeat(np.repeat(np.asarray(scales, np.float64), block_rows, 0)[:rows], BLOCK, 1)[:, :cols]


def tops(x, block_rows):
    """Largest finite magnitude of every block."""
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    r, c = blocks_of_rows(a.shape[0], block_rows), blocks(a.shape[1])
    wide = np.zeros((r * block_rows, c * BLOCK))
    wide[:a.shape[0], :a.shape[1]] = a
    return wide.reshape(r, block_rows, c, BLOCK).max((1, 3))


def blocks_of_rows(rows, block_rows):
    return -(-rows // block_rows)


def quantize(x, block_rows):
    """Codes and scales of fp32 values by the definition, every step rounded to fp32."""
    x = np.asarray(x, np.float32)
    top = tops(x, block_rows).astype(np.float32)
    scales = np.where(top == 0, np.float32(1), np.maximum(top / np.float32(TOP), np.float32(2.0 ** -126))).astype(np.float32)
    by = (np.float32(1) / scales).astype(np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        v = x * np.repeat(np.repeat(by, block_rows, 0)[:x.shape[0]], BLOCK, 1)[:, :x.shape[1]]
    return ofp8.e4m3_encode(np.where(np.isfinite(x), v, np.nan)), scales


def norm(x, add, gain, eps, offset):
    """(s, y) over the last axis."""
    s = np.asarray(x, np.float64) + (0.0 if add is None else np.asarray(add, np.float64))
    m = np.mean(s * s, -1, keepdims=True) + eps
    y = s * np.where(m == 0, 0.0, 1.0 / np.sqrt(np.where(m == 0, 1.0, m)))
    return s, y if gain is None else y * (np.asarray(gain, np.float64) + offset)


def norm_slack(channels):
    """How far y may be off, relative to it, before it is rounded to its type: s is off by one rounding (and its square by two); a lane adds 16 squares one
    after another, or 8 ceil(channels / 8192) of more than 16384 channels, and 6 + 16 more additions join the lanes; the mean, eps, the root (2 of its steps), 1 / root (half of
    what the sum is off), gain + offset and the two products.  In 64 bits gain + offset is exact, in 32 off by a rounding of the sum."""
    return ((max(16, 8 * -(-channels // 8192)) + 22 + 2 + 2) / 2 + 2 + 4) * U32


def act(z, gate):
    import torch
    return z / (1.0 + torch.exp(-z)) if gate == "silu" else z * (0.5 * (1.0 + torch.tanh((2.0 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3))))


def values64(codes, scales, block_rows):
    """What codes (uint8) and scales stand for, on the device that has them."""
    import torch
    table = torch.from_numpy(ofp8.e4m3_decode(np.arange(256))).to(codes.device)
    rows, cols = codes.shape
    return table[codes.long()] * scales.double().repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def product(av, wv, bias=None, gate=None, add=None, eight_bit=False):
    """(av wv^T and what follows, bound on what it may be off before it is rounded to its type): torch's elementary operations in 64 bits."""
    import torch
    c, size = av @ wv.t().contiguous(), av.abs() @ wv.t().abs().contiguous()
    K = av.shape[1]
    # a block's 128 products one after another, its scale (2 roundings) and addition, a few sums joined at the end
    off = (min(K, BLOCK) + blocks(K) + 3 + 16) * U32 * size
    if eight_bit:
        # the 8-bit instruction adds eight products (of columns 8 i .. 8 i + 7 of a block) at once, cutting each off at 2^-13 of the largest one's power of two
        for k in range(0, K, 8):
            top = torch.zeros_like(c)
            for e in range(k, min(k + 8, K)):
                top = torch.maximum(top, torch.outer(av[:, e].abs(), wv[:, e].abs()))
            off = off + 7 * 2.0 ** -13 * top
    if bias is not None:
        c = c + bias.double()
        off = off + U32 * c.abs()
    if gate is not None:
        f = c.shape[1] // 2
        z, u, dz, du = c[:, :f], c[:, f:], off[:, :f], off[:, f:]
        # act's slope is below 1.13; computed, act is off by 8 roundings of z at most (its exponential by its argument's, which weighs less the
        # smaller act is)
        a0 = act(z, gate)
        da = 1.13 * dz + 8 * U32 * z.abs()
        c, off = a0 * u, da * (u.abs() + du) + a0.abs() * du + 2 * U32 * (a0 * u).abs()
    if add is not None:
        c = c + add.double()
        off = off + U32 * c.abs()
    return c, off


def check_rounded(got, want, off, unit, what=""):
    """got, want, off: tensors or arrays; got is want to within off, rounded once."""
    got, want, off = (torch_of(x) for x in (got, want, off))
    bound = off + unit * (want.abs() + off)
    err = (got - want).abs()
    bad = ~(err <= bound) & ~(got.isnan() & want.isnan())
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst error / bound {float((err / bound.clamp(min=1e-300))[bad].max()):.3g} at {bad.nonzero()[0].tolist()}"


def torch_of(x):
    import torch
    return torch.from_numpy(np.asarray(x, np.float64)) if not hasattr(x, "data_ptr") else x.double()


def check_codes(codes, scales, want, off, what=""):
    """Codes (uint8) and scales of values that are `want` to within `off`."""
    import torch
    scales, want, off = (torch_of(x) for x in (scales, want, off))
    rows, cols = want.shape
    pad = lambda x: torch.nn.functional.pad(x, (0, -cols % BLOCK)).view(rows, -1, BLOCK)      # noqa: E731
    top, far = pad(torch.where(want.isfinite(), want.abs(), 0.0)).amax(2), pad(torch.where(off.isfinite(), off, 0.0)).amax(2)
    low = torch.where(top == 0, 1.0, (top / TOP).clamp(min=2.0 ** -126))
    exact_one = (top == 0) & (far == 0)
    assert (scales[exact_one] == 1.0).all(), what
    ok = (scales - low).abs() <= far / TOP + 2 * U32 * low + 2.0 ** -149
    assert (ok | exact_one).all(), f"{what}: scales off by {float(((scales - low).abs() / low).max()):.3g}"
    every = scales.repeat_interleave(BLOCK, 1)[:, :cols]
    value = values64(codes, scales, 1)
    # a code is off by half a step, of the smallest codes' 2^-9 at least; the fp32 factor and product by two roundings
    bound = off + U8 * (want.abs() + off) * (1 + 4 * U32) + 4 * U32 * want.abs() + 2.0 ** -10 * every
    bad = ~((value - want).abs() <= bound) & ~(value.isnan() & ~want.isfinite())
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} codes, worst {float(((value - want).abs() / bound)[bad].max()):.3g} at {bad.nonzero()[0].tolist()}"
