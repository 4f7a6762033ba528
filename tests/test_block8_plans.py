"""What a product's arguments lead to on the host: the instruction that sums, the tiles."""

import math
import os
import random
import shutil
import subprocess

import pytest

from block8_edges import EDGES
from block8_shapes import SHAPES
from paper_2504_02921_amd import binding as hb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """(kind, gate, rows, rows of w, columns) of many products -> (8-bit instruction, shape, its rows, shape of the rest, tiles, tiles of the rest, shapes) of each."""
    exe, csrc = str(tmp_path_factory.mktemp("plans") / "plans"), os.path.join(ROOT, "paper_2504_02921_amd", "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                        os.path.join(ROOT, "tests", "block8_plan_driver.cpp"), os.path.join(csrc, "hr_block8_host.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)          # the sanitizer runtime must come first in the link order

    def run(products):
        lines = "".join(f"{int(kind.startswith('block8'))} {hb.HR_BF16 if kind.startswith('bf16') else hb.HR_F32} {int(kind.endswith('fast'))} {gate} {m} {n} {k}\n"
                        for kind, gate, m, n, k in products)
        r = subprocess.run([exe], input=lines, capture_output=True, text=True, env=env)
        assert r.returncode == 0, (r.stdout + r.stderr)[-2000:]
        got = [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]
        assert len(got) == len(products)
        return got
    return run


def test_only_callers_that_ask_for_speed_get_the_8_bit_sums(plans):
    sizes = [(gate, m, n, k) for gate in (0, 1, 2) for m in (1, 20, 300, 12800) for n in (256, 6144) for k in (128, 4100)]
    for kind in ("bf16", "f32", "block8"):
        assert all(p[0] == 0 for p in plans([(kind, *s) for s in sizes])), kind
        assert all(p[0] == 1 for p in plans([(kind + " fast", *s) for s in sizes])), kind
    # bf16 results take the tiles of fp32 ones
    assert plans([("bf16", *s) for s in sizes]) == plans([("f32", *s) for s in sizes])


def test_neither_launch_of_a_product_has_more_tiles_than_a_launch_can(plans):
    """Rows behind the largest tiles are a second launch, with tiles of its own: a product whose first launch is accepted has no second one of too many."""
    most = (1 << 22) - 512
    sizes = [("bf16 fast", 0, 513, 181444029, 64), ("f32", 0, 513, 186746523, 1398), ("bf16", 0, 257, 372375436, 1834), ("f32 fast", 1, 518, 184733696, 15),
             ("f32", 0, 257, 836829046, 3934685), ("bf16 fast", 1, 513, 179889408, 6)]
    rng = random.Random(4)
    for _ in range(20000):
        gate, n = rng.choice((0, 1)), int(math.exp(rng.uniform(math.log(1 << 20), math.log(1 << 30))))
        sizes.append((rng.choice(("bf16", "f32", "f32 fast")), gate, rng.choice((257, 300, 513, 521, 1000, 3000)), max(n // 256 * 256, 256) if gate else n, rng.choice((16, 128, 700, 4000))))
    for size, (_, shape, rows, rest, tiles, rest_tiles, _) in zip(sizes, plans(sizes)):
        assert tiles > most or rest_tiles <= most, (size, shape, rows, rest, tiles, rest_tiles)


# Shapes in the host's order: groups along k, and workgroups at once where they take several tiles (else 0)
GROUPS = [8, 8, 8, 8, 4, 2, 1, 2, 1, 2, 1, 1, 2, 1, 1, 4, 2, 1, 1]
AT_ONCE = [0] * 11 + [512, 0, 0, 256] + [0] * 4
FEW = 2          # the first shapes have one kernel for both instructions


def classes(size, plan):
    """What the loop over k of a product's launches goes by: (kind, gate, shape, one, two, an odd (3) or even (4) number of turns, a second tile of a workgroup)."""
    kind, gate, k = size[0], size[1], size[4]
    _, shape, _, rest, tiles, rest_tiles, shapes = plan
    assert shapes == len(GROUPS) == len(AT_ONCE)
    for s, n in ((shape, tiles), (rest, rest_tiles)):
        if s >= 0:
            turns = -(-(-(-k // 128)) // GROUPS[s])
            yield "f32" if s < FEW else kind.replace("bf16", "f32"), gate, s, turns if turns < 3 else 3 + (turns % 2 == 0), 0 < AT_ONCE[s] < n


def test_every_way_through_the_loop_over_k_that_a_product_takes_is_tested(plans):
    """With columns that end inside 16, whose last codes are set to zero in LDS: the sizes that the GPU tests run have every class that sizes of all kinds do."""
    rng = random.Random(6)
    size = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi))))      # noqa: E731
    drawn = []
    for kind in ("f32", "f32 fast", "block8", "block8 fast"):
        for gate in (0, 1):
            for _ in range(5000):
                n, k = size(16, 30000), size(1, 5000)
                drawn.append((kind, gate, size(1, 30000), max(n // 256 * 256, 256) if gate else n, k + (k % 16 == 0)))
    sizes = [s for s in SHAPES + EDGES if s[4] % 16]
    taken = {c for s, p in zip(drawn, plans(drawn)) for c in classes(s, p)}
    tested = {c for s, p in zip(sizes, plans(sizes)) for c in classes(s, p)}
    assert taken <= tested, sorted(taken - tested)
