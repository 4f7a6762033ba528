"""The demo's layer of a caller's own against plain operations, with bounds that a wrong step passes."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,queries,window", [((40, 130), (5, 9), 64), ((200, 17, 64), (24, 1, 40), 16), ((1,), (3,), 1000)])
def test_the_demos_layer_is_what_plain_operations_give(lens, queries, window):
    """Attention: v is a projection of normed rows by normal deviates over the root of their number, so of deviates of size 1 (documents' values are smaller), below 6
    in all of some thousand; an output is a mean of them, off by its rounding to bf16 (2^-8), by its weights' to half (2^-11), and by fp32 sums, which the
    last 2^-11 is for.  Projections: E4M3 moves a value by half of a step of 2^-3 at most, 2^-4 / 3^0.5 = 0.036 of it or less in the mean; two operands, 0.051.  A gate's two
    factors are off by that each, the slope of silu being below 1.1: 0.076; with the rounding of the codes and of the next weights 0.092 of the branch, which is less of the stream."""
    import torch
    from paper_2504_02921_amd import binding as hb
    from paper_2504_02921_amd import demo, workloads
    cfg, rng = workloads.ModelCfg("layer", 1, 256, 4, 2, 64, 384, 500, 1e6, 1e-6, dtype="bf16"), np.random.default_rng(4)
    docs = [rng.integers(0, cfg.vocab, n).astype(np.int32) for n in lens]
    pool = hb.KVPool(1, cfg.n_kv_heads, cfg.head_dim, 32, "bf16", "cuda:0")
    model = hb.Model(cfg, workloads.SeededWeights(cfg, seed=1, std=0.05), "cuda:0")
    try:
        pages = [pool.alloc(-(-n // hb.PAGE_TOKENS)) for n in lens]
        model.doc_prefill(pool, docs, pages)
        gap, away = demo.layer_of_the_callers(pool, cfg, docs, pages, list(queries), window)
        torch.cuda.synchronize()
        assert gap < 6 * (2.0 ** -8 + 2.0 ** -10)
        assert 0.01 < away < 0.1                                         # 8 bits are not nothing
    finally:
        model.close()
        pool.close()
