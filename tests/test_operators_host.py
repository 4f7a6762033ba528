"""The operators for models whose layers the caller runs, on a machine without a GPU: frequencies, sizes, and every refusal that the host
makes before anything is enqueued."""

import ctypes as C
import math

import numpy as np
import pytest

from oracle import reranker as orr
from paper_2504_02921_amd import binding as hb

FAKE = 0x7F0000000000      # never dereferenced on the host


def pool_handle(kv="bf16", d=64, n_kv=2, pages=8, layers=2):
    cfg = hb.make_pool_cfg(layers, n_kv, d, pages, kv)
    st, h = hb.hr_kv_pool_create(cfg, FAKE, hb.hr_kv_pool_bytes(cfg))
    assert st == hb.HR_OK
    return h


# ---- frequencies --------------------------------------------------------------------------------------------------------
def test_plain_frequencies_are_the_oracles():
    f = hb.Rope(64, 1.0e6).freqs
    x = np.zeros((1, 1, 64))
    x[0, 0, :32] = 1.0
    y = orr.rope(x, np.array([7.0]), 1.0e6)[0, 0]
    np.testing.assert_allclose(np.cos(7.0 * f), y[:32], atol=1e-14)
    np.testing.assert_allclose(np.sin(7.0 * f), y[32:], atol=1e-14)


def test_scaled_frequencies():
    plain = hb.Rope(128, 500000.0).freqs
    np.testing.assert_allclose(hb.Rope(128, 500000.0, scaling="linear", factor=4.0).freqs, plain / 4.0, rtol=1e-15)
    base = hb.Rope(128, 500000.0, scaling="base", factor=4.0).freqs
    np.testing.assert_allclose(base, (500000.0 * 4.0 ** (128 / 126)) ** (-np.arange(64) / 64.0), rtol=1e-13)
    assert base[0] == 1.0 and abs(base[-1] * 4.0 / plain[-1] - 1.0) < 1e-12        # the fastest pair stays, the slowest is stretched whole
    bands = hb.Rope(128, 500000.0, scaling="bands", factor=8.0, original_len=8192, low=1.0, high=4.0).freqs
    turns = 8192 * plain / (2 * math.pi)
    np.testing.assert_array_equal(bands[turns >= 4], plain[turns >= 4])
    np.testing.assert_allclose(bands[turns <= 1], plain[turns <= 1] / 8.0, rtol=1e-15)
    between = (turns > 1) & (turns < 4)
    assert between.any() and np.all(bands[between] < plain[between]) and np.all(bands[between] > plain[between] / 8.0)
    ramp = hb.Rope(128, 500000.0, scaling="ramp", factor=16.0, original_len=4096, low=1.0, high=32.0)
    turns = 4096 * plain / (2 * math.pi)
    np.testing.assert_array_equal(ramp.freqs[turns > 40], plain[turns > 40])
    np.testing.assert_allclose(ramp.freqs[turns < 0.7], plain[turns < 0.7] / 16.0, rtol=1e-15)
    assert np.all(np.diff(ramp.freqs) < 0)
    assert abs(ramp.cfg.amplitude - (0.1 * math.log(16.0) + 1.0)) < 1e-6


@pytest.mark.parametrize("bad", [dict(head_dim=1), dict(head_dim=1025), dict(rotary_dim=3), dict(rotary_dim=66), dict(rotary_dim=0), dict(base=1.0),
                                 dict(base=float("nan")), dict(amplitude=0.0), dict(amplitude=float("inf")), dict(scaling="linear", factor=0.5),
                                 dict(scaling="base", rotary_dim=2, factor=2.0), dict(scaling="bands", factor=2.0, original_len=0.0),
                                 dict(scaling="ramp", factor=2.0, original_len=4096, low=4.0, high=4.0), dict(layout="spiral"), dict(scaling="more")])
def test_rope_configurations_that_are_refused(bad):
    with pytest.raises(hb.HrError) as e:
        hb.Rope(**{**dict(head_dim=64, base=10000.0), **bad})
    assert e.value.status == hb.HR_ERR_INVALID_ARG


def rope_call(cfg=None, freqs=None, dtype=hb.HR_BF16, tokens=5, positions=FAKE, first=0, period=0, n=1, **side):
    cfg = cfg or hb.hr_rope_cfg(64, 64, 0, 0, 1.0, 10000.0, 1.0, 0.0, 1.0, 4.0)
    freqs = np.full(cfg.rotary_dim // 2, 0.5) if freqs is None else freqs
    t = (hb.hr_rope_tensor * 2)()
    for s in t:
        s.in_, s.out, s.n_heads = FAKE, FAKE + 4096, 2
        s.in_token_stride, s.in_head_stride, s.out_token_stride, s.out_head_stride = 128, 64, 128, 64
    for k, v in side.items():
        setattr(t[0], k, v)
    return hb.lib.hr_rope_apply(C.byref(cfg), freqs.ctypes.data if freqs is not False else None, dtype, tokens, positions, first, period, t, n, 0, None)


def test_rope_calls_that_are_refused():
    bad, ok = hb.HR_ERR_INVALID_ARG, hb.HR_OK
    assert rope_call(tokens=0) == ok
    assert rope_call(freqs=np.full(32, 7.0)) == bad and rope_call(freqs=np.full(32, -0.1)) == bad and rope_call(freqs=np.full(32, np.nan)) == bad
    assert rope_call(dtype=hb.HR_FP8_E4M3) == bad and rope_call(tokens=-1) == bad and rope_call(n=0) == bad and rope_call(n=3) == bad
    assert rope_call(in_=None) == bad and rope_call(out=None) == bad and rope_call(n_heads=0) == bad
    assert rope_call(in_token_stride=-1) == bad and rope_call(out_token_stride=127) == bad and rope_call(out_head_stride=63) == bad
    assert rope_call(out_token_stride=64, out_head_stride=128) == bad                # token 2 of head 0 is token 0 of head 1
    assert rope_call(out=FAKE, out_token_stride=256) == bad                          # in place with other strides
    assert rope_call(out=FAKE + 1) == bad and rope_call(in_token_stride=1 << 60) == bad
    assert rope_call(positions=None, first=-1) == bad and rope_call(positions=None, period=-1) == bad
    assert rope_call(positions=None, first=2 ** 31 - 3) == hb.HR_ERR_LEN_RANGE       # tokens 0 .. 4
    assert rope_call(tokens=(1 << 30) + 1) == hb.HR_ERR_LEN_RANGE


# ---- tables and attention ---------------------------------------------------------------------------------------------------
def tables(pool, n_pairs=3, max_tokens=40, stride=4, n_q=8, **change):
    t = hb.hr_pair_tables(n_pairs, max_tokens, stride, n_q, *[FAKE + 4096 * i for i in range(8)],
                          hb.lib.hr_pair_tables_sched_bytes(pool, n_pairs, max_tokens, n_q))
    for k, v in change.items():
        setattr(t, k, v)
    return t


def build(pool, t, docs=None, pair_doc=FAKE, lens=FAKE):
    docs = docs or hb.hr_doc_list(2, 6, FAKE, FAKE, FAKE)
    return hb.lib.hr_pair_tables_build(pool, C.byref(docs), pair_doc, lens, C.byref(t), None)


def test_tables_that_are_refused():
    pool = pool_handle()
    bad = hb.HR_ERR_INVALID_ARG
    assert build(pool, tables(pool, n_pairs=0)) == hb.HR_OK
    for k in ("q_cu", "doc_lens", "page_table", "tok_pos", "tok_pair", "order", "report", "sched"):
        assert build(pool, tables(pool, **{k: None})) == bad
    assert build(pool, tables(pool, sched=FAKE + 4)) == bad
    assert build(pool, tables(pool, sched_bytes=64)) == hb.HR_ERR_WORKSPACE_SMALL
    assert build(pool, tables(pool, n_pairs=-1)) == bad and build(pool, tables(pool, max_tokens=-1)) == bad and build(pool, tables(pool, pt_stride=-1)) == bad
    assert build(pool, tables(pool, n_q_heads=7)) == bad                             # two kv heads
    assert build(pool, tables(pool, pt_stride=(1 << 26) + 1)) == hb.HR_ERR_LEN_RANGE
    assert build(pool, tables(pool, max_tokens=1 << 29)) == hb.HR_ERR_LEN_RANGE      # rows of a kv head: four times as many
    assert build(None, tables(pool)) == bad and build(pool, tables(pool), pair_doc=None) == bad and build(pool, tables(pool), lens=None) == bad
    assert build(pool, tables(pool), docs=hb.hr_doc_list(-1, 6, FAKE, FAKE, FAKE)) == bad
    assert build(pool, tables(pool), docs=hb.hr_doc_list(2, 6, None, FAKE, FAKE)) == bad
    assert build(pool, tables(pool), docs=hb.hr_doc_list(2, 6, FAKE, FAKE, None)) == bad
    assert hb.lib.hr_pair_tables_sched_bytes(pool, 3, 40, 7) == 0 and hb.lib.hr_pair_tables_sched_bytes(None, 3, 40, 8) == 0


def attend(pool, t, ws=FAKE, ws_bytes=None, dtype=hb.HR_BF16, layer=0, scale=0.0, cap=0.0, window=0, **change):
    a = hb.hr_attention_args(dtype, layer, scale, cap, window, FAKE, FAKE, FAKE, FAKE, None, None, None, 512, 64, 128, 64, 128, 64, 512, 64)
    for k, v in change.items():
        setattr(a, k, v)
    need = hb.lib.hr_pair_attention_workspace_bytes(pool, C.byref(t))
    return hb.lib.hr_pair_attention(pool, C.byref(t), C.byref(a), ws, need if ws_bytes is None else ws_bytes, None)


def test_attention_calls_that_are_refused():
    pool = pool_handle()
    t, bad = tables(pool), hb.HR_ERR_INVALID_ARG
    assert attend(pool, tables(pool, n_pairs=0)) == hb.HR_OK and attend(pool, tables(pool, max_tokens=0)) == hb.HR_OK
    assert attend(pool, t, dtype=hb.HR_F32) == hb.HR_ERR_MISMATCH and attend(pool_handle("f32"), t) == hb.HR_ERR_MISMATCH
    assert attend(pool, t, dtype=hb.HR_FP8_E4M3) == bad
    assert attend(pool, t, layer=2) == bad and attend(pool, t, layer=-1) == bad
    for k, v in (("scale", math.nan), ("scale", math.inf), ("cap", -1.0), ("cap", math.inf), ("cap", 1e-30), ("window", -1)):
        assert attend(pool, t, **{k: v}) == bad
    assert attend(pool, t, q=None) == bad and attend(pool, t, out=None) == bad and attend(pool, t, k=None) == bad and attend(pool, t, v=None) == bad
    assert attend(pool, t, q=FAKE + 1) == bad and attend(pool, t, out_token_stride=511) == bad and attend(pool, t, out_head_stride=60) == bad
    assert attend(pool, t, k_token_stride=-1) == bad and attend(pool, tables(pool, sched_bytes=16)) == hb.HR_ERR_WORKSPACE_SMALL
    long = tables(pool, n_pairs=1, max_tokens=1, stride=4096)
    need = hb.lib.hr_pair_attention_workspace_bytes(pool, C.byref(long))
    assert need > 0                                                                  # a long document's keys are cut into pieces
    assert attend(pool, long, ws_bytes=need - 1) == hb.HR_ERR_WORKSPACE_SMALL
    assert attend(pool, long, ws=None) == bad and attend(pool, long, ws=FAKE + 16) == bad


def test_the_work_list_has_room_for_every_distribution_of_the_tokens():
    """Blocks of 32 rows: however the tokens fall on documents, each one's last block alone is partly filled."""
    pool = pool_handle(n_kv=1, d=64)
    for n_pairs, max_tokens, g in ((1, 1, 1), (5, 3, 7), (40, 100, 7), (100, 40, 4), (7, 1000, 16)):
        ints = hb.lib.hr_pair_tables_sched_bytes(pool, n_pairs, max_tokens, g) // 4
        rng = np.random.default_rng(n_pairs)
        most = 0
        for _ in range(200):
            split = np.bincount(rng.integers(0, n_pairs, max_tokens), minlength=n_pairs)
            most = max(most, int((-(-split * g // 32)).sum()))
        assert max_tokens * g // 32 + min(n_pairs, max_tokens) >= most
        assert ints >= most * 8 + max_tokens * 4 + 6 * n_pairs


def test_one_tensors_output_is_not_the_others():
    cfg = hb.hr_rope_cfg(64, 64, 0, 0, 1.0, 10000.0, 1.0, 0.0, 1.0, 4.0)
    freqs = np.full(32, 0.5)

    def call(a, b, tokens=1):
        t = (hb.hr_rope_tensor * 2)(*[hb.hr_rope_tensor(x, y, 2, 128, 64, 128, 64) for x, y in (a, b)])
        return hb.lib.hr_rope_apply(C.byref(cfg), freqs.ctypes.data, hb.HR_BF16, tokens, FAKE, 0, 0, t, 2, 0, None)

    w, x, y, z = (FAKE + 4096 * i for i in range(4))
    for a, b in (((w, z), (x, z)), ((w, x), (x, y)), ((x, y), (w, x)), ((w, w), (w, w))):
        assert call(a, b) == hb.HR_ERR_INVALID_ARG
    assert call((w, w), (x, x), tokens=0) == hb.HR_OK


def test_calls_that_no_launch_can_hold_are_refused():
    # 64 heads of 1024 channels: a wavefront has one token
    wide = hb.hr_rope_cfg(1024, 256, 0, 0, 1.0, 10000.0, 1.0, 0.0, 1.0, 4.0)
    assert rope_call(cfg=wide, tokens=1 << 27, n_heads=1, in_token_stride=1024, in_head_stride=1024, out_token_stride=1024, out_head_stride=1024) == hb.HR_ERR_LEN_RANGE
    pool = pool_handle(n_kv=8)
    assert attend(pool, tables(pool, n_pairs=1 << 21, max_tokens=1 << 21, n_q=32), q_token_stride=2048, out_token_stride=2048) == hb.HR_ERR_LEN_RANGE


def test_numbers_that_would_wrap_around_are_refused():
    for x in (-1, 1 << 31, (1 << 32) + 5):
        with pytest.raises(hb.HrError):
            hb._int32(x, "x")
    assert hb._int32((1 << 31) - 1, "x") == (1 << 31) - 1
    class Pool:                                             # noqa: E306
        mem = type("M", (), {"device": "cpu"})
    for change in (dict(n_pairs=1 << 32), dict(max_tokens=(1 << 32) + 4), dict(pt_stride=-1), dict(n_q_heads=1 << 31)):
        with pytest.raises(hb.HrError):
            hb.PairTables(Pool(), **{**dict(n_pairs=1, max_tokens=1, pt_stride=1, n_q_heads=1), **change})
