"""The operators for models whose layers the caller runs, where sizes, masks and values come to an end: odd heads, large caps, rows of NaN, outputs
over inputs, tiles in pieces.  References and bounds are those of operators_ref.py."""

import numpy as np
import pytest

import operators_ref as R
from test_gpu_operators import DEV, Batch, check_rope, dev_i32, dtype_of, hb, to64, torch

pytestmark = pytest.mark.gpu


# ---- rotary positions ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,r", [(65, 32), (33, 2), (97, 64), (3, 2), (129, 128), (259, 6), (64, 30)])
def test_rope_of_odd_heads_stays_inside_them(kind, layout, d, r):
    """Heads that another array's values follow, in the input and in the output."""
    T = torch()
    heads, tokens = 3, 7
    gen = T.Generator().manual_seed(d)
    x = T.randn((tokens, heads, d), generator=gen).to(dtype_of(kind)).to(DEV)
    pos = np.random.default_rng(d).integers(0, 5000, tokens)
    rope = hb().Rope(d, 10000.0, rotary_dim=r, layout=layout)
    y, = rope.apply(dev_i32(pos), x)
    check_rope(y, x, pos, rope, layout, kind)
    assert T.equal(y[..., r:], x[..., r:])
    wide = T.full((tokens, heads, d + 1), 3.0, dtype=x.dtype, device=DEV)
    rope.apply(dev_i32(pos), x, out=[wide[..., :d]])
    assert T.equal(wide[..., :d], y) and bool((wide[..., d] == 3.0).all())
    wide[..., :d] = x
    rope.apply(dev_i32(pos), wide[..., :d], out=[wide[..., :d]])
    assert T.equal(wide[..., :d], y) and bool((wide[..., d] == 3.0).all())
