"""The operators of a layer's projections in 8 bits: the root-mean-square norm with the residual's addition (and 8-bit codes with scales beside or
instead of its output), codes with scales made of rows and of weights, and the product of two such matrices with what follows it in a layer.

An 8-bit matrix is E4M3 codes and fp32 scales, value = code * scale: one scale for each row and 128 of its columns (activations), or for each
tile of 128 x 128 (weights).  `run` computes the operators in plain torch operations, or, with `own` set, with the calls of the library.  Shapes
are those of workloads.MODELS (0.5B: hidden 896, feed-forward 4864; 8B: hidden 4096, feed-forward 14336, 32 + 2 x 8 heads of 128)."""

import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 128
TOP = 448.0          # the largest E4M3 value
PITCH = 16           # bytes that a row of codes is padded to


# ---- cases ----------------------------------------------------------------------------------------------------------
def _norm(tokens, heads, channels, dtype, add, y, block8, offset=0.0, **more):
    """heads > 1: every head of a token is normed for itself, q's rows of a fused projection.  y, block8: which outputs; add: a residual stream."""
    return dict(op="norm", tokens=tokens, heads=heads, channels=channels, dtype=dtype, add=add, y=y, block8=block8, offset=offset, **more)


def _quantize(rows, cols, block_rows, dtype, **more):
    return dict(op="quantize", rows=rows, cols=cols, block_rows=block_rows, dtype=dtype, **more)


def _product(m, n, k, out, gate="none", bias=False, add=False, **more):
    """n: rows of the weights; a gate halves them: act(first half) * second half."""
    return dict(op="product", m=m, n=n, k=k, out=out, gate=gate, bias=bias, add=add, **more)


def listed():
    return [
        # the shortest request, five candidates and a query of 13 tokens, 0.5B shape: the stream's sum and the next projection's codes
        _norm(65, 1, 896, "bf16", True, False, True, name="norm_request_0p5b"),
        # the same for a batch of 400 pairs at the 8B shape
        _norm(12800, 1, 4096, "bf16", True, False, True, name="norm_batch_8b"),
        # heads of q normed one by one before rotary positions, a long batch
        _norm(25600, 32, 128, "bf16", False, True, False, name="norm_heads_8b"),
        # an fp32 stream of an odd width, gains kept as their distance from 1
        _norm(1000, 1, 5003, "f32", True, True, False, 1.0, name="norm_odd_f32"),
        # a model's gate and up weights on their way into 8 bits
        _quantize(28672, 4096, 128, "bf16", name="quantize_weight_8b"),
        # rows that attention left in fp32
        _quantize(777, 4864, 1, "f32", name="quantize_rows_0p5b"),
        # one token through the q, k and v projection of the 8B shape: the weights' bytes
        _product(1, 6144, 4096, "bf16", name="product_single_8b"),
        # the shortest request's down projection, 0.5B shape, onto the residual stream: latency
        _product(65, 896, 4864, "bf16", add=True, name="product_request_0p5b"),
        # gate and up of a few tokens, into the codes that the down projection reads
        _product(20, 28672, 4096, "block8", gate="silu", name="product_gate_few_8b"),
        # odd sizes throughout, fp32 out
        _product(777, 1003, 2500, "f32", bias=True, name="product_ragged"),
        # the down projection of a batch onto the residual stream
        _product(12800, 4096, 14336, "bf16", add=True, name="product_down_batch_8b"),
        # the largest: gate and up of that batch
        _product(12800, 28672, 4096, "block8", gate="silu", name="product_gate_batch_8b"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Multiples of 128, of 16, and any."""
    step = rng.choice((128, 128, 16, 1))
    return max(lo, _log_int(rng, lo, hi) // step * step)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("norm", "quantize", "product", "product"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if op == "norm":
            if rng.random() < 0.3:
                c = _norm(_log_int(rng, 1, 25600), rng.choice((2, 5, 8, 14, 32)), rng.choice((64, 80, 96, 128, 256)), dtype, False, True, False,
                          rng.choice((0.0, 1.0)))
            else:
                y = rng.random() < 0.6
                c = _norm(_log_int(rng, 1, 25600), 1, _width(rng, 64, 16384), dtype, rng.random() < 0.7, y, not y or rng.random() < 0.4, rng.choice((0.0, 1.0)))
        elif op == "quantize":
            c = _quantize(_log_int(rng, 1, 32768), _width(rng, 64, 16384), rng.choice((1, 128)), dtype)
        else:
            out = rng.choice(("bf16", "bf16", "f32", "block8"))
            gate = rng.choice(("none", "none", "silu", "gelu"))
            n = _width(rng, 16, 32768)
            if gate != "none":
                n = max(n // 256 * 256, 256)
            c = _product(_log_int(rng, 1, 25600), n, _width(rng, 32, 16384), out, gate, rng.random() < 0.3, out != "block8" and rng.random() < 0.4)
        if _cost(c) <= most:
            return c


# ---- sizes ----------------------------------------------------------------------------------------------------------
def _esz(dtype):
    return {"f32": 4.0, "bf16": 2.0}[dtype]


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    c = case
    if c["op"] == "norm":
        values, esz = float(c["tokens"]) * c["heads"] * c["channels"], _esz(c["dtype"])
        moved = values * esz * (1 + (2 if c["add"] else 0) + (1 if c["y"] else 0)) + 4.0 * c["channels"]
        if c["block8"]:
            moved += values + 4.0 * c["tokens"] * _blocks(c["channels"])
        return {"bytes": moved, "flops": 4.0 * values}
    if c["op"] == "quantize":
        values = float(c["rows"]) * c["cols"]
        rows = c["rows"] if c["block_rows"] == 1 else _blocks(c["rows"])
        return {"bytes": values * (_esz(c["dtype"]) + 1.0) + 4.0 * rows * _blocks(c["cols"]), "flops": 2.0 * values}
    m, n, k = float(c["m"]), float(c["n"]), float(c["k"])
    wide = n if c["gate"] == "none" else n / 2
    size = 1.0 if c["out"] == "block8" else _esz(c["out"])
    moved = (m + n) * k + 4.0 * m * _blocks(c["k"]) + 4.0 * _blocks(c["n"]) * _blocks(c["k"]) + m * wide * size * (2 if c["add"] else 1)
    moved += (4.0 * n if c["bias"] else 0.0) + (4.0 * m * _blocks(int(wide)) if c["out"] == "block8" else 0.0)
    return {"bytes": moved, "flops": 2.0 * m * n * k}


def _cost(c):
    w = work(c)
    return w["flops"] / 2e15 + w["bytes"] / 4e12


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _tdt(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _activations(rows, cols, gen):
    """Rows of a residual stream or of a layer's inside: of many sizes, some channels much larger than the others."""
    x = torch.randn((rows, cols), generator=gen, device=DEV)
    channel = torch.randn(cols, generator=gen, device=DEV).mul_(0.5).exp_()
    channel = torch.where(torch.rand(cols, generator=gen, device=DEV) < 0.01, channel * 20.0, channel)
    return x.mul_(channel).mul_(torch.randn((rows, 1), generator=gen, device=DEV).mul_(0.5).exp_())


def _codes_in_hand(x, block_rows):
    """Codes and scales as a program has them, in rows of a whole number of 16 bytes."""
    codes, scales = _in_blocks(x, block_rows)
    held = torch.zeros((x.shape[0], -(-x.shape[1] // PITCH) * PITCH), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    held[:, :x.shape[1]] = codes
    return held[:, :x.shape[1]], scales


def _inputs(case, seed):
    c = case
    gen = torch.Generator(DEV)
    gen.manual_seed(seed)
    if c["op"] == "norm":
        st = dict(case=c, add=None, gain=torch.randn(c["channels"], generator=gen, device=DEV).mul_(0.2).add_(1.0 - c["offset"]))
        if c["heads"] > 1:       # q of a fused projection, whose k and v lie behind it
            rows = torch.randn((c["tokens"], (c["heads"] + 2) * c["channels"]), generator=gen, device=DEV).to(_tdt(c["dtype"]))
            return st | dict(x=rows[:, :c["heads"] * c["channels"]].unflatten(1, (c["heads"], c["channels"])))
        st["x"] = _activations(c["tokens"], c["channels"], gen).to(_tdt(c["dtype"]))
        if c["add"]:             # the stream, and what a layer adds to it
            st["add"] = torch.randn((c["tokens"], c["channels"]), generator=gen, device=DEV).to(_tdt(c["dtype"]))
        return st
    if c["op"] == "quantize":
        make = _activations if c["block_rows"] == 1 else lambda r, k, g: torch.randn((r, k), generator=g, device=DEV).mul_(0.02)
        return dict(case=c, x=make(c["rows"], c["cols"], gen).to(_tdt(c["dtype"])))
    st = dict(case=c, bias=None, add=None)
    st["a"], st["a_scales"] = _codes_in_hand(_activations(c["m"], c["k"], gen), 1)
    st["w"], st["w_scales"] = _codes_in_hand(torch.randn((c["n"], c["k"]), generator=gen, device=DEV).mul_(0.02), BLOCK)
    if c["bias"]:
        st["bias"] = torch.randn(c["n"], generator=gen, device=DEV)
    if c["add"]:
        wide = c["n"] if c["gate"] == "none" else c["n"] // 2
        st["add"] = torch.randn((c["m"], wide), generator=gen, device=DEV).to(_tdt(c["out"]))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own and case["op"] == "product":
        from paper_2504_02921_amd import binding as hb
        st["a8"], st["w8"] = hb.Block8(st["a"], st["a_scales"]), hb.Block8(st["w"], st["w_scales"], block_rows=BLOCK)
    return st


# ---- the operators --------------------------------------------------------------------------------------------------
def _tiles(x, block_rows):
    """[rows / block_rows][block_rows][columns / 128][128], zeros behind the last row and column."""
    r, k = -x.shape[0] % block_rows, -x.shape[1] % BLOCK
    if r or k:
        x = torch.nn.functional.pad(x, (0, k, 0, r))
    return x.view(x.shape[0] // block_rows, block_rows, x.shape[1] // BLOCK, BLOCK)


def _in_blocks(x, block_rows):
    """Codes of float32 values and their scales: the largest magnitude of a block becomes 448."""
    t = _tiles(x, block_rows)
    top = t.abs().amax((1, 3))
    scales = torch.where(top > 0, top / TOP, 1.0)
    codes = (t / scales[:, None, :, None]).clamp_(-TOP, TOP).to(torch.float8_e4m3fn)
    return codes.view(t.shape[0] * block_rows, -1)[:x.shape[0], :x.shape[1]], scales


def _values(codes, scales, block_rows):
    """The float32 values that codes and scales stand for."""
    t = _tiles(codes.float(), block_rows)
    return t.mul(scales[:, None, :, None]).view(t.shape[0] * block_rows, -1)[:codes.shape[0], :codes.shape[1]]


def _plain_norm(st):
    c, x = st["case"], st["x"].float()
    if c["add"]:
        x = x + st["add"].float()
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * (st["gain"] + c["offset"])
    got = [x.to(_tdt(c["dtype"]))] if c["add"] else []
    if c["y"]:
        got.append(y.to(_tdt(c["dtype"])))
    return got + list(_in_blocks(y, 1)) if c["block8"] else got


def _gated(first, second, gate):
    if gate == "silu":
        return first / (1.0 + torch.exp(-first)) * second
    return 0.5 * first * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (first + 0.044715 * first * first * first))) * second


def _plain_product(st):
    c = st["case"]
    y = torch.matmul(_values(st["a"], st["a_scales"], 1), _values(st["w"], st["w_scales"], BLOCK).t())
    if c["bias"]:
        y = y + st["bias"]
    if c["gate"] != "none":
        y = _gated(y[:, :c["n"] // 2], y[:, c["n"] // 2:], c["gate"])
    if c["add"]:
        y = y + st["add"].float()
    return list(_in_blocks(y, 1)) if c["out"] == "block8" else [y.to(_tdt(c["out"]))]


def _own(st):
    from paper_2504_02921_amd import binding as hb
    c = st["case"]
    if c["op"] == "norm":
        y, total, block8 = hb.rms_norm(st["x"], st["gain"], add=st["add"], eps=1e-6, gain_offset=c["offset"], out=c["y"], total=c["add"], block8=c["block8"])
        got = [t for t in (total, y) if t is not None]
        return got + [block8.codes, block8.scales] if c["block8"] else got
    if c["op"] == "quantize":
        q = hb.block_quantize(st["x"], block_rows=c["block_rows"])
        return [q.codes, q.scales]
    gate = None if c["gate"] == "none" else c["gate"]
    if c["out"] == "block8":
        q = hb.block_matmul(st["a8"], st["w8"], gate=gate, bias=st["bias"], block8=True)
        return [q.codes, q.scales]
    return [hb.block_matmul(st["a8"], st["w8"], dtype=_tdt(c["out"]), gate=gate, bias=st["bias"], add=st["add"])]


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["op"] == "quantize":
        return list(_in_blocks(state["x"].float(), c["block_rows"]))
    return _plain_norm(state) if c["op"] == "norm" else _plain_product(state)


# ---- the definitions, in 64 bits --------------------------------------------------------------------------------------
def _exact_codes(x, block_rows):
    """What codes would be without their rounding, and the scales."""
    rows, cols = x.shape
    down, across = torch.arange(rows, device=DEV) // block_rows, torch.arange(cols, device=DEV) // BLOCK
    wide = torch.zeros((rows, int(across[-1]) + 1), dtype=torch.float64, device=DEV)
    for b in range(wide.shape[1]):
        wide[:, b] = x[:, b * BLOCK:(b + 1) * BLOCK].abs().max(1).values
    top = torch.zeros((int(down[-1]) + 1, wide.shape[1]), dtype=torch.float64, device=DEV)
    top = top.index_reduce_(0, down, wide, "amax") / TOP
    scales = top + (top == 0).double()
    return [x / scales[down].repeat_interleave(BLOCK, 1)[:, :cols], scales]


def _exact_matrix(codes, scales, block_rows):
    value = codes.double()
    for b in range(scales.shape[1]):
        value[:, b * BLOCK:(b + 1) * BLOCK] *= scales[:, b].double().repeat_interleave(block_rows)[:codes.shape[0], None]
    return value


def exact(case, seed):
    c, st = case, _inputs(case, seed)
    if c["op"] == "quantize":
        return _exact_codes(st["x"].double(), c["block_rows"])
    if c["op"] == "norm":
        x = st["x"].double() + (st["add"].double() if c["add"] else 0.0)
        size = torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["channels"] + 1e-6)
        y = (st["gain"].double() + c["offset"]) * (x / size)
        return ([x] if c["add"] else []) + ([y] if c["y"] else []) + (_exact_codes(y, 1) if c["block8"] else [])
    a, w = _exact_matrix(st["a"], st["a_scales"], 1), _exact_matrix(st["w"], st["w_scales"], BLOCK).t().contiguous()
    y = a @ w
    if c["bias"]:
        y += st["bias"].double()
    if c["gate"] != "none":
        g, up = y.chunk(2, 1)
        turned = torch.sigmoid(g) if c["gate"] == "silu" else torch.sigmoid(math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3))
        y = g * turned * up                                  # (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
    if c["add"]:
        y = y + st["add"].double()
    return _exact_codes(y, 1) if c["out"] == "block8" else [y]
