"""The operators of a layer's projections in 8 bits on a machine without a GPU: every refusal that the host makes before anything is enqueued."""

import ctypes as C
import math
import os
import random
import shutil
import subprocess

import pytest

from block8_shapes import SHAPES
from paper_2504_02921_amd import binding as hb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FAKE = 0x7F0000000000      # never dereferenced on the host
BAD, LONG, MISMATCH = hb.HR_ERR_INVALID_ARG, hb.HR_ERR_LEN_RANGE, hb.HR_ERR_MISMATCH
KINDS = ("bf16", "f32", "f32 fast", "block8", "block8 fast")
NAN, INF = float("nan"), float("inf")


def block8(n, k, per=1, at=1, **more):
    b = hb.hr_block8(FAKE + at * 0x10000000, FAKE + at * 0x10000000 + 0x8000000, n, k, per, -(-k // 16) * 16, -(-k // 128))
    for k, v in more.items():
        setattr(b, k, v)
    return b


# ---- norm
def norm(block8=None, **more):
    a = hb.hr_norm_args(hb.HR_BF16, 1, 64, 1e-6, 0.0, 0, FAKE, None, None, FAKE + 4096, None, None, 64, 64, 64, 64, 64, 64, 64, 64)
    a.tokens = 4 if "tokens" not in more else more.pop("tokens")
    for k, v in more.items():
        setattr(a, k, v)
    if block8 is not None:
        a.block8 = C.pointer(block8)
    return hb.lib.hr_rms_norm(C.byref(a), None)


def test_norms_that_are_refused():
    assert hb.lib.hr_rms_norm(None, None) == BAD
    assert norm(tokens=0) == hb.HR_OK and norm(tokens=0, x=None) == hb.HR_OK
    for bad in (dict(dtype=hb.HR_FP8_E4M3), dict(heads=0), dict(heads=65537), dict(channels=0), dict(channels=65537), dict(tokens=-1), dict(eps=-1e-9), dict(eps=NAN),
                dict(eps=INF), dict(gain_offset=NAN), dict(x=None), dict(x=FAKE + 1), dict(out=None), dict(out=FAKE + 4097), dict(gain=FAKE + 2), dict(total=FAKE + 1),
                dict(add=FAKE + 1), dict(x_token_stride=-64), dict(x_token_stride=1 << 60), dict(out_token_stride=63), dict(out_token_stride=0), dict(heads=2, out_head_stride=63),
                dict(heads=2, out_token_stride=100), dict(out=FAKE, out_token_stride=65), dict(total=FAKE + 4096), dict(gain=FAKE + 4096), dict(total=FAKE, total_token_stride=80),
                dict(add=FAKE + 8192, total=FAKE + 8192, add_token_stride=70)):
        assert norm(**bad) == BAD, bad
    assert norm(tokens=(1 << 30) + 1) == LONG
    for bad in (dict(codes=FAKE + 8), dict(codes=None), dict(scales=None), dict(row_stride=72), dict(row_stride=48), dict(row_stride=(1 << 22) + 16), dict(scale_stride=0), dict(block_rows=128),
                dict(codes=FAKE), dict(scales=FAKE), dict(scales=FAKE + 4096), dict(rows=-1), dict(cols=0), dict(scales=FAKE + 0x20000002)):
        assert norm(block8(4, 64, **bad)) == BAD, bad
    b = block8(4, 64)
    b.scales = b.codes
    assert norm(b) == BAD and norm(block8(4, 128), heads=2) == BAD
    assert norm(block8(5, 64)) == MISMATCH and norm(block8(4, 65)) == MISMATCH
    assert norm(block8(4, (1 << 22) + 1, row_stride=1 << 22)) == LONG


# ---- codes
def quantize(out, dtype=hb.HR_F32, x=FAKE, stride=64):
    return hb.lib.hr_block_quantize(dtype, x, stride, C.byref(out) if out is not None else None, None)


def test_codes_that_are_refused():
    assert quantize(block8(0, 64), x=None) == hb.HR_OK
    assert quantize(None) == BAD and quantize(block8(4, 64), dtype=hb.HR_FP8_E4M3) == BAD and quantize(block8(4, 64), x=None) == BAD
    assert quantize(block8(4, 64), x=FAKE + 2) == BAD and quantize(block8(4, 64), stride=-1) == BAD and quantize(block8(4, 64, block_rows=64)) == BAD
    assert quantize(block8(4, 64, codes=FAKE)) == BAD and quantize(block8(4, 64, scales=FAKE)) == BAD and quantize(block8(4, 64, scales=FAKE + 0x10000000)) == BAD
    assert quantize(block8((1 << 30) + 1, 64)) == LONG and quantize(block8(1 << 30, 1024, 128), stride=1024) == LONG


# ---- product
def product(a=None, w=None, out8=None, **more):
    a, w = a or block8(4, 100), w or block8(256, 100, 128, at=2)
    m = hb.hr_matmul_args(hb.HR_BF16, 0, 0, None, None, FAKE + 64, 256, 256, None)
    if out8 is not None:
        m.block8, m.out = C.pointer(out8), None
    for k, v in more.items():
        setattr(m, k, v)
    return hb.lib.hr_block_matmul(C.byref(a), C.byref(w), C.byref(m), None)


def test_products_that_are_refused():
    a, w = block8(4, 100), block8(256, 100, 128, at=2)
    assert hb.lib.hr_block_matmul(None, C.byref(w), None, None) == BAD and hb.lib.hr_block_matmul(C.byref(a), None, None, None) == BAD
    assert hb.lib.hr_block_matmul(C.byref(a), C.byref(w), None, None) == BAD
    assert product(block8(0, 100)) == hb.HR_OK and product(w=block8(0, 100, 128, at=2)) == hb.HR_OK
    for bad in (dict(dtype=hb.HR_FP8_E4M3), dict(gate=3), dict(gate=-1), dict(out=None), dict(out=FAKE + 1), dict(add=FAKE + 1), dict(bias=FAKE + 2), dict(out_stride=255),
                dict(out_stride=0), dict(add=FAKE + 64, add_stride=300), dict(add=FAKE, add_stride=-1), dict(bias=FAKE + 64), dict(out=a.codes), dict(out=w.scales), dict(out=a.scales), dict(out=w.codes)):
        assert product(**bad) == BAD, bad
    assert product(w=a) == BAD and product(a=w) == BAD and product(a=block8(4, 100, row_stride=100)) == BAD and product(a=block8(4, 100, codes=FAKE + 4)) == BAD
    assert product(a=block8(4, 101)) == MISMATCH and product(w=block8(384, 100, 128, at=2), gate=1) == MISMATCH and product(w=block8(250, 100, 128, at=2), gate=2) == MISMATCH
    assert product(block8(1 << 30, 100), block8(1 << 29, 100, 128, at=2), out_stride=1 << 29) == LONG
    good = lambda **more: block8(4, 256, at=3, **more)      # noqa: E731
    assert product(out8=good(), out=FAKE + 64) == BAD and product(out8=good(), add=FAKE) == BAD and product(out8=good(codes=a.codes)) == BAD
    assert product(out8=good(scales=w.scales)) == BAD and product(out8=good(block_rows=128)) == BAD
    assert product(out8=block8(4, 128, at=3)) == MISMATCH and product(out8=block8(5, 256, at=3)) == MISMATCH and product(out8=good(), gate=1) == MISMATCH
    assert product(block8(0, 100), out8=block8(0, 256, at=3)) == hb.HR_OK


def test_products_of_more_tiles_than_a_launch_has_are_refused():
    """A launch counts its lanes in 32 bits: 2^22 workgroups, of 1024 lanes where they are widest, are too many."""
    assert product(block8(1, 100), block8(1 << 30, 100, 128, at=2), out_stride=1 << 30) == LONG
    assert product(block8(1 << 30, 100), block8(256 * 256, 100, 128, at=2), out_stride=1 << 16) == LONG
    assert product(block8(0, 100), block8(1 << 30, 100, 128, at=2), out_stride=1 << 30) == hb.HR_OK


@pytest.mark.parametrize("what", ["codes", "scales"])
def test_matrices_on_the_host_are_refused_before_the_device_is_asked(what):
    import torch
    with pytest.raises(hb.HrError):
        hb.rms_norm(torch.zeros((4, 64)))
    with pytest.raises(hb.HrError):
        hb.block_quantize(torch.zeros((4, 64)))
    q = hb.Block8.empty(4, 64, device="cpu")
    with pytest.raises(hb.HrError):
        hb.block_matmul(q, hb.Block8.empty(128, 64, 128, device="cpu"))
    with pytest.raises(hb.HrError):
        hb.Block8(*((q.codes[:, :32], torch.zeros((4, 2))) if what == "codes" else (q.codes, q.scales.double())))
    with pytest.raises(hb.HrError):
        hb.Block8.empty(1 << 31, 64, device="cpu")


def test_a_matrix_keeps_its_tensors():
    """Calls take the places that the matrix began with, so its tensors cannot be replaced under it."""
    import torch
    q = hb.Block8(torch.zeros((4, 64), dtype=torch.uint8), torch.ones((4, 1)))
    for name in ("codes", "scales"):
        with pytest.raises(AttributeError):
            setattr(q, name, getattr(q, name).clone())
    assert q.c.codes == q.codes.data_ptr() and q.c.scales == q.scales.data_ptr()
    w = hb.Block8(torch.zeros((128, 64), dtype=torch.uint8), torch.ones((1, 1)), 128)
    for pair in ((q.codes, w), (q, w.codes), (None, w)):
        with pytest.raises(hb.HrError):
            hb.block_matmul(*pair)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_shape_of_tile_that_a_product_takes_is_tested(tmp_path):
    """The host's choice of tiles, with AddressSanitizer + UBSan: for sizes of all kinds it ends, and what it takes is among what the GPU tests run."""
    exe, csrc = str(tmp_path / "shapes"), os.path.join(ROOT, "paper_2504_02921_amd", "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                        os.path.join(ROOT, "tests", "block8_shapes_driver.cpp"), os.path.join(csrc, "hr_block8_host.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    rng = random.Random(1)
    size = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi))))      # noqa: E731
    drawn = [(kind, gate, size(1, 60000), max(size(16, 60000) // 256 * 256, 256) if gate else size(16, 60000), size(32, 32768))
             for kind in KINDS for gate in (0, 1) for _ in range(3000)]
    drawn += [(kind, gate, m, n, k) for kind in KINDS for gate in (0, 1) for m in (1, 1 << 30) for n in (256, (1 << 30) - 256) for k in (1, 1 << 22)]
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)          # the sanitizer runtime must come first in the link order
    lines = "".join(f"{int(kind.startswith('block8'))} {int(kind == 'bf16' or kind.endswith('fast'))} {gate} {m} {n} {k}\n" for kind, gate, m, n, k in drawn + SHAPES)
    r = subprocess.run([exe], input=lines, capture_output=True, text=True, env=env)
    assert r.returncode == 0, (r.stdout + r.stderr)[-2000:]
    plans = [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]
    assert len(plans) == len(drawn) + len(SHAPES)
    taken = {(d[0], d[1], p[0]) for d, p in zip(drawn, plans)}
    tested = {(d[0], d[1], p[0]) for d, p in zip(SHAPES, plans[len(drawn):])}
    assert taken <= tested, sorted(taken - tested)
    assert {d[0] for d, p in zip(SHAPES, plans[len(drawn):]) if p[1] >= 0} == set(KINDS)
