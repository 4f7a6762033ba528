"""The operators for models whose layers the caller runs, through the Python entry points, against 64-bit references (operators_ref.py)
with bounds derived there."""

import numpy as np
import pytest

from oracle import fp8 as ofp8
from oracle import reranker as orr

import operators_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def hb():
    from paper_2504_02921_amd import binding
    return binding


def torch():
    import torch
    return torch


def dev_i32(a):
    return torch().from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def to64(t):
    return t.detach().to(torch().float64).cpu().numpy()


def dtype_of(kind):
    return torch().float32 if kind == "f32" else torch().bfloat16


# ---- rotary positions ---------------------------------------------------------------------------------------------------
def check_rope(y, x, pos, rope, layout, kind, inverse=False):
    want, size = R.rope(to64(x), pos, rope.freqs, layout, rope.cfg.amplitude, inverse)
    unit = R.U32 if kind == "f32" else R.UBF
    # one rounding; sine and cosine off by the fp32 remainder of the angle, their series and the amplitude, the products and sum by theirs
    bound = unit * np.abs(want) + 8 * R.U32 * size
    err = np.abs(to64(y) - want)
    assert np.all(err <= bound), f"max err / bound {np.max(err / np.maximum(bound, 1e-300)):.3f}"


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,r,heads,tokens", [(64, 64, 14, 65), (128, 128, 40, 3), (64, 32, 4, 17), (80, 20, 5, 9), (96, 6, 3, 130), (256, 256, 2, 5), (34, 34, 1, 1),
                                              (2, 2, 1, 70), (1024, 250, 1, 2)])
def test_rope_rotates_by_the_formula(kind, layout, d, r, heads, tokens):
    T = torch()
    gen = T.Generator().manual_seed(d + r + heads)
    x = T.randn((tokens, heads, d), generator=gen).to(dtype_of(kind)).to(DEV)
    pos = np.random.default_rng(d).integers(0, 1 << 20, tokens)
    rope = hb().Rope(d, 10000.0, rotary_dim=r, layout=layout)
    y, = rope.apply(dev_i32(pos), x)
    check_rope(y, x, pos, rope, layout, kind)
    assert T.equal(y[..., r:], x[..., r:])                                      # what is not rotated is copied


def test_rope_far_positions_frequencies_and_amplitude():
    T = torch()
    x = T.randn((4, 3, 128), generator=T.Generator().manual_seed(1)).to(DEV)
    pos = np.array([0, 1, (1 << 24) + 1, (1 << 31) - 1])
    for rope in (hb().Rope(128, 500000.0, scaling="bands", factor=8.0, original_len=8192), hb().Rope(128, 10000.0, scaling="ramp", factor=32.0, original_len=4096, high=32.0),
                 hb().Rope(128, 10000.0, freqs=np.linspace(0.0, 6.2, 64), amplitude=0.25)):
        y, = rope.apply(dev_i32(pos[:3]), x[:3])
        check_rope(y, x[:3], pos[:3], rope, "half", "f32")
        # at 2^31 an angle's fp64 product is off by up to 2^-22 turns: looked at alone, with that added
        y, = rope.apply(dev_i32(pos), x)
        want, size = R.rope(to64(x), pos, rope.freqs, "half", rope.cfg.amplitude)
        assert np.all(np.abs(to64(y) - want) <= (8 * R.U32 + 2 * np.pi * 2.0 ** -21) * size + R.U32 * np.abs(want))


def test_rope_two_tensors_strides_in_place_inverse_and_positions_of_its_own():
    T, H = torch(), hb()
    gen = T.Generator().manual_seed(2)
    rows = T.randn((37, 14 + 2 + 2, 64), generator=gen).to(T.bfloat16).to(DEV)
    q, k, v = rows[:, :14], rows[:, 14:16], rows[:, 16:]
    q0, k0, v0 = q.clone(), k.clone(), v.clone()
    rope = H.Rope(64, 1.0e6)
    pos = np.arange(37) % 10 + 500
    yq, yk = rope.apply(500, q, k, period=10)
    check_rope(yq, q0, pos, rope, "half", "bf16")
    check_rope(yk, k0, pos, rope, "half", "bf16")
    rope.apply(dev_i32(pos), q, k, out=[q, k])                                  # in place, in rows that hold v too
    assert T.equal(q, yq) and T.equal(k, yk) and T.equal(v, v0)
    # head-major, one element off, back again
    base = T.zeros(3 * 37 * 64 + 1, dtype=T.float32, device=DEV)
    x = base[1:].view(3, 37, 64).transpose(0, 1)
    x.copy_(T.randn((37, 3, 64), generator=gen))
    x0 = x.clone()
    y, = rope.apply(dev_i32(pos), x)
    back, = rope.apply(dev_i32(pos), y, inverse=True)
    check_rope(back, y, pos, rope, "half", "f32", inverse=True)
    assert float((back - x0).abs().max()) < 1e-5
    # a token without a position is left out
    pos2 = pos.copy()
    pos2[[0, 5, 36]] = -1
    out = T.full_like(x0, 7.0)
    rope.apply(dev_i32(pos2), x0, out=[out])
    assert bool((out[[0, 5, 36]] == 7.0).all()) and T.equal(out[1:5], y[1:5])
    z, = rope.apply(dev_i32(np.zeros(0)), x0[:0])
    assert z.shape == (0, 3, 64)


def test_rope_refuses_wrong_tensors():
    T, H = torch(), hb()
    rope = H.Rope(64, 1.0e6)
    x = T.zeros((4, 2, 64), device=DEV, dtype=T.bfloat16)
    p = dev_i32(np.arange(4))
    for call in (lambda: rope.apply(p.long(), x), lambda: rope.apply(p[:3], x), lambda: rope.apply(p.cpu(), x), lambda: rope.apply(p, x.half()), lambda: rope.apply(p, x.cpu()),
                 lambda: rope.apply(p, x[..., :32]), lambda: rope.apply(p, x.transpose(0, 2)), lambda: rope.apply(p, x, x, x), lambda: rope.apply(p, x, x[:3]),
                 lambda: rope.apply(p, x, x.float()), lambda: rope.apply(p, x, out=[x[:, :1]]), lambda: rope.apply(p, x, out=[x[:1].expand(4, 2, 64)])):
        with pytest.raises(H.HrError):
            call()


# ---- tables -----------------------------------------------------------------------------------------------------------------
def corpus(rng, lens):
    cu = np.concatenate([[0], np.cumsum(-(-np.maximum(lens, 0) // R.PAGE))]).astype(np.int64)
    return cu, rng.permutation(int(cu[-1])).astype(np.int32)


def built(pool, num_pages, lens, cu, pages, pair_doc, q_lens, max_tokens, stride, n_q=14):
    H = hb()
    t = H.PairTables(pool, len(pair_doc), max_tokens, stride, n_q_heads=n_q)
    for x in (t.q_cu, t.doc_lens, t.page_table, t.tok_pos, t.tok_pair, t.order, t.report, t.sched):
        x.fill_(-77)
    t.build(H.DocList(dev_i32(lens), dev_i32(cu), dev_i32(pages)), dev_i32(pair_doc), dev_i32(q_lens))
    want = R.tables(lens, cu, pages, num_pages, pair_doc, q_lens, max_tokens, stride)
    for name, w in want.items():
        np.testing.assert_array_equal(getattr(t, name).cpu().numpy(), w, err_msg=name)
    return t, want


@pytest.mark.parametrize("n_pairs,n_docs,q_hi,spare", [(1, 1, 1, 0), (1, 3, 40, 9), (20, 60, 32, 0), (63, 2, 5, 100), (64, 64, 1, 0), (65, 300, 3, 1), (1000, 1, 9, 3),
                                                       (1025, 255, 20, 0), (4097, 256, 12, 5000), (5000, 70000, 7, 1), (9000, 400, 0, 16)])
def test_tables_are_the_references(n_pairs, n_docs, q_hi, spare):
    rng = np.random.default_rng(n_pairs + n_docs)
    lens = rng.integers(0, 100, n_docs)
    cu, pages = corpus(rng, lens)
    pool = hb().KVPool(1, 2, 16, max(len(pages), 1), "bf16", DEV)
    q_lens = rng.integers(0, q_hi + 1, n_pairs)
    built(pool, len(pages), lens, cu, pages, rng.integers(-1, n_docs, n_pairs), q_lens, int(q_lens.sum()) + spare, 7)


@pytest.mark.parametrize("n_pairs,n_docs", [(256, 40), (257, 40), (2048, 3), (4999, 40), (5000, 40), (16000, 40000), (16000, 60000), (65535, 500), (65536, 500), (300, 140000)])
def test_tables_of_batches_on_either_side_of_a_choice(n_pairs, n_docs):
    rng = np.random.default_rng(n_pairs)
    lens = rng.integers(0, 40, n_docs)
    cu, pages = corpus(rng, lens)
    pool = hb().KVPool(1, 2, 16, len(pages), "bf16", DEV)
    q_lens = rng.integers(0, 4, n_pairs)
    built(pool, len(pages), lens, cu, pages, rng.integers(-1, n_docs, n_pairs), q_lens, int(q_lens.sum()) + 2, 3)


@pytest.mark.parametrize("docs", ["one", "two", "a long one between short ones", "all different", "none", "the last ones"])
def test_tables_of_pairs_spread_unevenly(docs):
    n, n_docs = 11000, 20000
    rng = np.random.default_rng(12)
    pair_doc = {"one": np.full(n, 7), "two": rng.integers(3, 5, n), "none": np.full(n, -1), "all different": rng.permutation(n), "the last ones": n_docs - 1 - rng.integers(0, 2, n),
                "a long one between short ones": np.where(rng.random(n) < 0.6, 500, rng.integers(400, 600, n))}[docs]
    lens = rng.integers(0, 40, n_docs)
    cu, pages = corpus(rng, lens)
    pool = hb().KVPool(1, 2, 16, len(pages), "bf16", DEV)
    q_lens = rng.integers(0, 4, n)
    built(pool, len(pages), lens, cu, pages, pair_doc, q_lens, int(q_lens.sum()) - 5, 3)


def test_work_lists_do_not_depend_on_the_way_they_are_built():
    """In one small workgroup, sorted and counted: the attention of the same pairs is the same, bit for bit."""
    T, H = torch(), hb()
    rng = np.random.default_rng(8)
    b = Batch("bf16", 14, 2, 64, [100, 0, 33, 300], rng.integers(-1, 4, 40), rng.integers(0, 9, 40), seed=8)
    want, log = b.check()
    for more, pairs in ((0, 260), (0, 6000), (30000, 11000)):      # empty pairs behind them, documents that nobody asks for
        lens = np.concatenate([b.doc_lens, np.zeros(more, np.int64)])
        cu, pages = corpus(np.random.default_rng(8), lens)
        t = H.PairTables(b.pool, 40 + pairs, b.tokens, 19, n_q_heads=14)
        t.build(H.DocList(dev_i32(lens), dev_i32(cu), b.list.tensors[2]), dev_i32(np.concatenate([b.pair_doc, np.full(pairs, -1)])),
                dev_i32(np.concatenate([b.q_lens, np.zeros(pairs, np.int64)])))
        out, log2 = H.pair_attention(b.pool, b.layer, t, b.q, b.k, b.v, with_lse=True)
        assert T.equal(out[:b.tokens], want[:b.tokens]) and T.equal(log2[:b.tokens], log[:b.tokens])


@pytest.mark.parametrize("n_pairs,n_docs", [(20, 50), (3000, 400), (12000, 9000)])
def test_tables_recorded_and_replayed(n_pairs, n_docs):
    """Built in one small workgroup, sorted and counted: replays with other documents and lengths, eager work between."""
    T, H = torch(), hb()
    rng = np.random.default_rng(n_pairs)
    lens = rng.integers(0, 60, n_docs)
    cu, pages = corpus(rng, lens)
    pool = H.KVPool(1, 2, 16, len(pages), "bf16", DEV)
    room = 6 * n_pairs
    listed, doc, q = H.DocList(dev_i32(lens), dev_i32(cu), dev_i32(pages)), dev_i32(np.zeros(n_pairs)), dev_i32(np.zeros(n_pairs))
    t, side, graph = H.PairTables(pool, n_pairs, room, 4, n_q_heads=14), T.cuda.Stream(), T.cuda.CUDAGraph()
    T.cuda.synchronize()
    with T.cuda.stream(side):
        t.build(listed, doc, q)
    side.synchronize()
    with T.cuda.graph(graph):
        t.build(listed, doc, q)
    for _ in range(4):
        pair_doc, q_lens = rng.integers(-1, n_docs, n_pairs), rng.integers(0, 7, n_pairs)
        doc.copy_(dev_i32(pair_doc))
        q.copy_(dev_i32(q_lens))
        graph.replay()
        T.cuda.synchronize()
        for name, w in R.tables(lens, cu, pages, len(pages), pair_doc, q_lens, room, 4).items():
            np.testing.assert_array_equal(getattr(t, name).cpu().numpy(), w, err_msg=name)


def test_tables_of_pairs_that_are_in_order_already():
    rng = np.random.default_rng(4)
    lens = rng.integers(1, 200, 50)
    cu, pages = corpus(rng, lens)
    pool = hb().KVPool(1, 2, 16, len(pages), "bf16", DEV)
    q = rng.integers(1, 30, 500)
    built(pool, len(pages), lens, cu, pages, np.sort(rng.integers(-1, 50, 500)), q, int(q.sum()), 13)


def test_tables_mend_and_report_what_is_wrong():
    rng = np.random.default_rng(5)
    lens = np.array([40, 300, 16, -5, 33])
    cu, pages = corpus(rng, lens)
    pool = hb().KVPool(1, 2, 16, len(pages), "bf16", DEV)
    n = len(pages)
    run = lambda **k: built(pool, n, **{**dict(lens=np.maximum(lens, 0), cu=cu, pages=pages, pair_doc=np.array([1, 0, 4]), q_lens=np.array([3, 2, 5]),  # noqa: E731
                                              max_tokens=10, stride=19), **k})[1]["report"][2]
    assert run() == 0
    assert run(pair_doc=np.array([1, 5, -2])) == 1
    assert run(q_lens=np.array([3, -2, 5])) == 2
    assert run(max_tokens=6) == 2 and run(max_tokens=0) == 2
    assert run(q_lens=np.array([2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1])) == 2
    assert run(stride=18) == 4 and run(stride=0) == 4
    assert run(lens=lens, pair_doc=np.array([3, 0, 4])) == 4
    assert run(lens=np.array([40, 301 + 16, 16, 0, 33])) == 4
    assert run(cu=np.array([0, 3, 2, 10 ** 6, 10 ** 6, -9])) == 4
    assert run(pages=np.where(np.arange(n) == 4, n, pages)) == 8
    assert run(pages=np.where(np.arange(n) == 4, -3, pages), pair_doc=np.array([1, 5, 0]), q_lens=np.array([3, 2, 6])) == 8 + 2 + 1


# ---- attention ---------------------------------------------------------------------------------------------------------------
class Batch:
    """A pool with documents, a batch of pairs, and the same in 64 bits."""

    def __init__(self, kv, n_q, n_kv, d, doc_lens, pair_doc, q_lens, seed=0, layers=2, layer=1, stride=None, spare=0, q_size=2.0):
        T, H = torch(), hb()
        rng = np.random.default_rng(seed)
        self.kv, self.n_q, self.n_kv, self.d, self.layer = kv, n_q, n_kv, d, layer
        self.doc_lens, self.pair_doc, self.q_lens = np.asarray(doc_lens), np.asarray(pair_doc), np.asarray(q_lens)
        cu, pages = corpus(rng, self.doc_lens)
        self.pool = H.KVPool(layers, n_kv, d, max(len(pages), 1), kv, DEV)
        self.docs = []
        for i, D in enumerate(self.doc_lens):
            D = int(D)
            k, v = (rng.standard_normal((layers, D, n_kv, d)) for _ in range(2))
            if D == 0:
                self.docs.append((np.zeros((0, n_kv, d)), np.zeros((0, n_kv, d))))
                continue
            ids = pages[cu[i]:cu[i + 1]]
            if kv == "fp8":
                (kc, ks), (vc, vs) = ofp8.quantize_doc_kv(k), ofp8.quantize_doc_kv(v)
                self.pool.write(D, ids, *[T.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in (kc, vc, ks.astype(np.float32), vs.astype(np.float32))])
                per = np.arange(D) // R.PAGE
                self.docs.append(tuple(ofp8.e4m3_decode(c)[layer] * s.astype(np.float32)[layer][per][:, :, None] for c, s in ((kc, ks), (vc, vs))))
            else:
                kt, vt = (T.from_numpy(x).to(dtype_of(kv)) for x in (k, v))
                self.pool.write(D, ids, kt.to(DEV), vt.to(DEV))
                self.docs.append((to64(kt[layer]), to64(vt[layer])))
        tokens = int(self.q_lens.sum())
        self.tokens = tokens
        stride = stride or max(1, int(-(-max(self.doc_lens, default=0) // R.PAGE)))
        self.tables = H.PairTables(self.pool, len(self.pair_doc), tokens + spare, stride, n_q_heads=n_q)
        self.list = H.DocList(dev_i32(self.doc_lens), dev_i32(cu), dev_i32(pages))
        self.tables.build(self.list, dev_i32(self.pair_doc), dev_i32(self.q_lens))
        gen = T.Generator().manual_seed(seed)
        rows = lambda heads, size: (T.randn((tokens + spare, heads, d), generator=gen) * size).to(dtype_of(kv)).to(DEV)  # noqa: E731
        self.q, self.k, self.v = rows(n_q, q_size), rows(n_kv, 1.0), rows(n_kv, 1.0)
        T.cuda.synchronize()

    def run(self, own=True, q=None, k=None, v=None, **a):
        H = hb()
        k, v = (self.k if k is None else k, self.v if v is None else v) if own else (None, None)
        return H.pair_attention(self.pool, self.layer, self.tables, self.q if q is None else q, k, v, with_lse=True, **a)

    def check(self, own=True, q=None, k=None, v=None, what="", **a):
        out, lse = self.run(own, q, k, v, **a)
        return self.compare(out, lse, own, q, k, v, what, **a)

    def compare(self, out, lse, own=True, q=None, k=None, v=None, what="", **a):
        n = self.tokens
        x = [to64(y if t is None else t)[:n] for t, y in ((q, self.q), (k, self.k), (v, self.v))]
        want, log, tol, tol_log = R.attention(x[0], x[1] if own else None, x[2] if own else None, self.docs, self.pair_doc, self.q_lens, scale=a.get("scale"),
                                              cap=a.get("cap", 0.0), slopes=None if a.get("slopes") is None else to64(a["slopes"]), window=a.get("window", 0),
                                              prefix=None if a.get("prefix_lens") is None else a["prefix_lens"].cpu().numpy(), pool=self.kv)
        got, got_log = to64(out)[:n], to64(lse)[:n]
        fine = np.isfinite(want)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
        np.testing.assert_array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)], err_msg=what)
        err = np.abs(got[fine] - want[fine])
        assert np.all(err <= tol[fine]), f"{what}: out, max err / bound {np.max(err / np.maximum(tol[fine], 1e-300)):.2f}"
        empty = log == -np.inf
        np.testing.assert_array_equal(got_log == -np.inf, empty, err_msg=what)
        err = np.abs(got_log[~empty] - log[~empty])
        assert np.all(err <= tol_log[~empty]), f"{what}: log-sum, max err / bound {np.max(err / tol_log[~empty]):.2f}"
        return out, lse


SHAPES = [("bf16", 14, 2, 64), ("bf16", 8, 2, 128), ("fp8", 6, 2, 64), ("fp8", 8, 1, 128), ("f32", 4, 4, 64), ("f32", 6, 1, 80), ("bf16", 3, 1, 96), ("fp8", 4, 2, 32),
          ("bf16", 2, 2, 16), ("f32", 2, 1, 256), ("bf16", 5, 1, 256), ("fp8", 34, 1, 112)]
# documents that end in, at and behind a page and a sub-tile; queries of no, one and many tokens; documents shared out of order, and none
DOCS = [1, 15, 16, 17, 31, 32, 33, 0, 64, 100, 300]
PAIRS = [10, 0, 1, -1, 2, 3, 10, 4, 5, 6, -1, 7, 8, 9, 10, 0]
LENS = [5, 1, 3, 2, 33, 1, 70, 0, 4, 1, 9, 6, 1, 2, 1, 8]


@pytest.mark.parametrize("kv,n_q,n_kv,d", SHAPES)
def test_attention_is_the_reference(kv, n_q, n_kv, d):
    T = torch()
    b = Batch(kv, n_q, n_kv, d, DOCS, PAIRS, LENS, seed=d, spare=3)
    slopes = T.exp2(-T.arange(1, n_q + 1).float() * 8 / n_q).to(DEV)
    prefix = dev_i32(np.arange(len(PAIRS)) * 2 - 3)                            # negative, shorter and longer than the query
    b.check(what="plain")
    b.check(scale=0.3, cap=5.0, what="cap")
    b.check(slopes=slopes, what="slopes")
    b.check(prefix_lens=prefix, what="prefix")
    for w in (1, 20, 33, 1000):
        b.check(window=w, what=f"window {w}")
        b.check(own=False, window=w, what=f"window {w}, documents only")         # rows that see nothing
    b.check(own=False, what="documents only")
    b.check(cap=30.0, slopes=slopes, prefix_lens=prefix, window=40, scale=-0.1, what="all")


@pytest.mark.parametrize("kv,n_q,n_kv,d", [("bf16", 14, 2, 64), ("fp8", 32, 8, 128), ("bf16", 8, 1, 128), ("f32", 4, 4, 64)])
@pytest.mark.parametrize("pairs,doc,query", [(1, 3000, 1), (2, 5000, 3), (40, 200, 1), (30, 70, 40), (70, 500, 37)])
def test_attention_of_few_and_of_many_rows(kv, n_q, n_kv, d, pairs, doc, query):
    """Few rows behind long documents (their keys in pieces), single tokens, many rows."""
    T = torch()
    rng = np.random.default_rng(pairs)
    b = Batch(kv, n_q, n_kv, d, rng.integers(doc // 2, doc + 1, pairs), rng.permutation(pairs), np.full(pairs, query), seed=3, layers=1, layer=0)
    b.check(what="plain")
    b.check(cap=20.0, what="cap")
    b.check(slopes=T.full((n_q,), 0.002, device=DEV), what="slopes")
    b.check(cap=30.0, slopes=T.full((n_q,), 0.01, device=DEV), scale=-0.1, own=False, what="cap and slopes")
    b.check(window=doc // 3, cap=20.0, slopes=T.full((n_q,), 0.01, device=DEV), what="edges inside a piece")
    b.check(own=False, window=2, what="pieces that see nothing")


@pytest.mark.parametrize("kv,d", [("bf16", 64), ("fp8", 128), ("f32", 64)])
def test_attention_of_one_document_for_all(kv, d):
    b = Batch(kv, 8, 2, d, [1500, 40], [0] * 60 + [1] * 3 + [0] * 9, np.random.default_rng(1).integers(0, 12, 72), seed=9)
    slopes = torch().full((8,), 0.003, device=DEV)
    b.check()
    b.check(cap=10.0, slopes=slopes, prefix_lens=dev_i32(np.arange(72) % 9))
    b.check(window=700)


@pytest.mark.parametrize("kv,d", [("bf16", 64), ("bf16", 128), ("fp8", 128), ("f32", 64)])
def test_what_is_not_seen_does_not_count(kv, d):
    """NaN and infinities in tokens that a row does not see: later ones, those behind the window, other pairs', rows of nobody, and keys of a
    document behind the length that the list gives it."""
    T, H = torch(), hb()
    n_q, n_kv = 4, 2
    b = Batch(kv, n_q, n_kv, d, [50, 20], [0, 1, 0, -1], [9, 4, 7, 40], seed=1, spare=5)
    q, k, v = b.q.clone(), b.k.clone(), b.v.clone()
    for t in (q, k, v):
        t[b.tokens:] = float("nan")
    v[4, 0, 3], v[4, 1, d - 1], v[11, 0, 5] = float("inf"), float("nan"), float("-inf")
    v[30, 1], v[40, 1, 7] = float("inf"), float("-inf")
    b.check(q=q, k=k, v=v, what="values")
    b.check(q=q, k=k, v=v, window=6, what="values, window")
    out, _ = b.run(q=q, k=k, v=v)
    q2, k2 = q.clone(), k.clone()
    q2[2], k2[15] = float("nan"), float("nan")                                   # a query row; a key that its pair's later tokens see
    bad, _ = b.run(q=q2, k=k2, v=v)
    hit = np.zeros(b.tokens, bool)
    hit[2], hit[15:20] = True, True
    assert bool(T.isnan(bad[:b.tokens][T.from_numpy(hit)]).all())
    keep = T.from_numpy(~hit).to(DEV)
    np.testing.assert_array_equal(to64(bad[:b.tokens][keep]), to64(out[:b.tokens][keep]))
    # a document of 50 tokens whose last 9 are not finite, given as one of 41
    if kv == "fp8":
        return
    kd, vd = (T.randn((2, 50, n_kv, d)).to(dtype_of(kv)) for _ in range(2))
    kd[:, 41:], vd[:, 41:] = float("nan"), float("inf")
    ids = np.arange(4, dtype=np.int32)
    pool = H.KVPool(2, n_kv, d, 4, kv, DEV)
    pool.write(50, ids, kd.to(DEV), vd.to(DEV))
    c = Batch(kv, n_q, n_kv, d, [41], [0, 0], [3, 30], seed=4)
    c.pool, c.docs = pool, [(to64(kd[1, :41]), to64(vd[1, :41]))]
    c.tables = H.PairTables(pool, 2, 33, 3, n_q_heads=n_q).build(H.DocList(dev_i32([41]), dev_i32([0, 4]), dev_i32(ids)), dev_i32([0, 0]), dev_i32([3, 30]))
    c.check(what="document cut")


@pytest.mark.parametrize("kv,n_q,n_kv", [("bf16", 12, 4), ("fp8", 6, 2)])
def test_attention_of_96_channels(kv, n_q, n_kv):
    """A head size whose rows are not a power of two: every shape and mask of the tests above."""
    test_attention_is_the_reference(kv, n_q, n_kv, 96)
    for pairs, doc, query in ((1, 3000, 1), (2, 5000, 3), (40, 200, 1), (30, 70, 40), (70, 500, 37)):
        test_attention_of_few_and_of_many_rows(kv, n_q, n_kv, 96, pairs, doc, query)
    test_attention_of_one_document_for_all(kv, 96)
    test_what_is_not_seen_does_not_count(kv, 96)


def test_attention_takes_views_and_leaves_other_rows_alone():
    T, H = torch(), hb()
    for kv, d in (("bf16", 64), ("bf16", 128), ("f32", 64)):
        b = Batch(kv, 6, 2, d, [40, 333], [1, 0, 1, 1], [5, 40, 1, 2], seed=6, spare=7)
        n = b.q.shape[0]
        flat = T.zeros(n * 10 * d + 1, dtype=b.q.dtype, device=DEV)
        rows = flat[1:].view(n, 10, d)                                          # packed rows that start one element off
        rows[:, :6], rows[:, 6:8], rows[:, 8:] = b.q, b.k, b.v
        out, lse = b.run()
        rows[b.tokens:] = float("nan")
        wide = T.full((8, n, d + 4), 3.0, dtype=b.q.dtype, device=DEV)
        into = wide[1:7, :, :d].transpose(0, 1)                                # head by head, rows apart
        got, lse2 = b.run(q=rows[:, :6], k=rows[:, 6:8], v=rows[:, 8:], out=into)
        assert got is into and T.equal(got[:b.tokens], out[:b.tokens]) and T.equal(lse[:b.tokens], lse2[:b.tokens])
        assert bool((into[b.tokens:] == 3.0).all()) and bool((wide[0] == 3.0).all()) and bool((wide[7] == 3.0).all()) and bool((wide[:, :, d:] == 3.0).all())


def test_attention_gives_the_same_bits_again_and_on_other_streams():
    T = torch()
    batches = [Batch("bf16", 14, 2, 64, [700, 200], [0, 1, 0, 1, 1], [20, 3, 1, 50, 9], seed=7), Batch("fp8", 8, 2, 128, [4000], [0], [2], seed=8)]
    first = [b.run() for b in batches]
    T.cuda.synchronize()
    streams = [T.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        again = [b.run(stream=s) for b, s in zip(batches, streams)]             # two calls at once
        T.cuda.synchronize()
        for x, y in zip(first, again):
            assert T.equal(x[0], y[0]) and T.equal(x[1], y[1])


@pytest.mark.parametrize("n_q,n_kv,d,q_len", [(14, 2, 64, 40), (32, 8, 128, 300), (14, 2, 64, 1200)])
def test_attention_of_fp8_keys_below_the_normal_range(n_q, n_kv, d, q_len):
    """Codes without an exponent count for what they are, in blocks and in tiles: 2^-9 steps beside a channel of 448 that the queries do not look at."""
    T = torch()
    D = 100
    b = Batch("fp8", n_q, n_kv, d, [D], [0], [q_len], seed=6)
    rng = np.random.default_rng(6)
    (_, _), (vc, vs) = [ofp8.quantize_doc_kv(rng.standard_normal((2, D, n_kv, d))) for _ in range(2)]
    kc = (rng.integers(0, 8, (2, D, n_kv, d)) | rng.integers(0, 2, (2, D, n_kv, d)) << 7).astype(np.uint8)
    kc[..., 0] = 0x7E
    ks = np.ones_like(vs)
    ids = b.list.tensors[2].cpu().numpy()
    b.pool.free(ids)
    b.pool.write(D, ids, *[T.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in (kc, vc, ks.astype(np.float32), vs.astype(np.float32))])
    per = np.arange(D) // R.PAGE
    b.docs[0] = tuple(ofp8.e4m3_decode(c)[b.layer] * s.astype(np.float32)[b.layer][per][:, :, None] for c, s in ((kc, ks), (vc, vs)))
    q = b.q * 256.0
    q[..., 0] = 0.0
    b.check(False, q=q)
    b.check(False, q=q, cap=5.0)


def test_attention_of_bad_tables_stays_in_the_pool():
    """Page ids outside the pool are -1 in the table; such a pair's rows are undefined, the others are as ever."""
    T, H = torch(), hb()
    b = Batch("bf16", 14, 2, 64, [100, 100], [0, 1], [4, 4], seed=2)
    want, _ = b.run()
    cu, pages = b.list.tensors[1], b.list.tensors[2].clone()
    pages[:3] = T.tensor([1 << 30, -5, 14], dtype=T.int32)
    b.tables.build(H.DocList(b.list.tensors[0], cu, pages), dev_i32([0, 1]), dev_i32([4, 4]))
    got, _ = b.run()
    assert T.equal(got[4:], want[4:]) and int(b.tables.report[2]) == H.TABLES_BAD_PAGE


def test_attention_refuses_wrong_tensors():
    T, H = torch(), hb()
    b = Batch("bf16", 4, 2, 64, [20], [0], [3], seed=0)
    for a in (dict(q=b.q[:2]), dict(q=b.q.float()), dict(q=b.q.cpu()), dict(q=b.q[..., :32]), dict(k=b.q), dict(out=b.q[:, :2]), dict(slopes=T.zeros(3, device=DEV)),
              dict(slopes=T.zeros(4)), dict(prefix_lens=T.zeros(1, dtype=T.int64, device=DEV)), dict(cap=-1.0), dict(scale=float("nan")), dict(window=-1)):
        with pytest.raises(H.HrError):
            b.run(**a)
    with pytest.raises(H.HrError):
        H.pair_attention(b.pool, 0, b.tables, b.q, b.k, None)
    with pytest.raises(H.HrError):
        H.pair_attention(b.pool, 2, b.tables, b.q)


# ---- together --------------------------------------------------------------------------------------------------------------
def layer_inputs(seed, kv, n_q, n_kv, d, tokens):
    T = torch()
    gen = T.Generator().manual_seed(seed)
    return (T.randn((tokens, n_q + 2 * n_kv, d), generator=gen) * 1.5).to(dtype_of(kv)).to(DEV)


@pytest.mark.parametrize("kv,n_q,n_kv,d,tol", [("f32", 4, 2, 64, 2e-5), ("bf16", 14, 2, 64, 3e-2), ("bf16", 8, 2, 128, 3e-2)])
def test_a_layer_of_rotary_positions_pool_tables_and_attention_is_the_oracles(kv, n_q, n_kv, d, tol):
    """Documents' keys rotated and written into the pool, tables from lengths, queries rotated at the tables' positions, attention: against the
    oracle's own rotary positions and attention on the unrotated values.  bf16: keys and queries are rounded once more on the way (2^-8 of values
    up to 6, in scores of up to 15: errors up to 2^-8 x 15 in a score, so some 3e-2 in outputs of size 1)."""
    T, H = torch(), hb()
    lens, pair_doc, q_lens = [37, 130, 5], [1, 0, 1, 2], [6, 1, 20, 3]
    cu, pages = corpus(np.random.default_rng(0), np.array(lens))
    pool = H.KVPool(1, n_kv, d, len(pages), kv, DEV)
    rope = H.Rope(d, 10000.0)
    raw = []
    for i, D in enumerate(lens):
        x = layer_inputs(i, kv, 0, n_kv, d, D)
        k, v = x[:, :n_kv], x[:, n_kv:].contiguous()
        raw.append((to64(k), to64(v)))
        pool.write(D, pages[cu[i]:cu[i + 1]], rope.apply(0, k)[0][None], v[None])
    tables = H.PairTables(pool, 4, sum(q_lens), 9, n_q_heads=n_q).build(H.DocList(dev_i32(lens), dev_i32(cu), dev_i32(pages)), dev_i32(pair_doc), dev_i32(q_lens))
    x = layer_inputs(10, kv, n_q, n_kv, d, sum(q_lens))
    q, k = rope.apply(tables.tok_pos, x[:, :n_q], x[:, n_q:n_q + n_kv])
    out = to64(H.pair_attention(pool, 0, tables, q, k, x[:, n_q + n_kv:]))
    t = 0
    for doc, n in zip(pair_doc, q_lens):
        D, y = lens[doc], to64(x[t:t + n])
        pos = D + np.arange(n)
        want = orr.prefix_causal_attention(orr.rope(y[:, :n_q], pos, 10000.0), orr.rope(raw[doc][0], np.arange(D), 10000.0), raw[doc][1],
                                           orr.rope(y[:, n_q:n_q + n_kv], pos, 10000.0), y[:, n_q + n_kv:])
        assert np.abs(out[t:t + n] - want).max() <= tol
        t += n


def test_calls_that_would_be_taken_for_others_are_refused():
    T, H = torch(), hb()
    b = Batch("bf16", 14, 2, 64, [40], [0], [3])
    other = H.KVPool(2, 2, 64, 8, "bf16", DEV)
    with pytest.raises(H.HrError):
        H.pair_attention(other, 0, b.tables, b.q, b.k, b.v)
    for a in (dict(scale=0.0), dict(window=(1 << 32) + 1), dict(window=-1)):
        with pytest.raises(H.HrError):
            b.run(**a)
    rope = H.Rope(64)
    for pos, a in ((1 << 32, {}), (-1, {}), (0, dict(period=(1 << 32) + 1))):
        with pytest.raises(H.HrError):
            rope.apply(pos, b.q, **a)
    with pytest.raises(H.HrError):
        rope.apply(0, b.q, b.q, out=[b.q, b.q])
    y, = rope.apply(np.int64(5), b.q)
    z, = rope.apply(5, b.q)
    assert T.equal(y, z)


def test_a_recorded_layer_replays_with_new_lengths_and_values():
    """Tables, rotary positions and attention recorded into two graphs, replayed in turn with other lengths, documents and values in the same
    buffers, with eager work between: the eager calls' bits every time."""
    T, H = torch(), hb()
    n_q, n_kv, d, pairs, room = 14, 2, 64, 6, 80
    rope = H.Rope(d, 10000.0)
    lens = np.array([200, 33, 5000, 64])
    cu, pages = corpus(np.random.default_rng(1), lens)
    graphs = []
    for g in range(2):
        b = Batch("bf16", n_q, n_kv, d, lens, [0], [1], seed=g)
        s = dict(pool=b.pool, list=b.list, tables=H.PairTables(b.pool, pairs, room, 313, n_q_heads=n_q), doc=dev_i32(np.zeros(pairs)), q_lens=dev_i32(np.ones(pairs)),
                 rows=T.zeros((room, n_q + 2 * n_kv, d), dtype=T.bfloat16, device=DEV), layer=b.layer)

        def chain(s=s, tables=None):
            t = (tables or s["tables"]).build(s["list"], s["doc"], s["q_lens"])
            q, k = rope.apply(t.tok_pos, s["rows"][:, :n_q], s["rows"][:, n_q:n_q + n_kv])
            return H.pair_attention(s["pool"], s["layer"], t, q, k, s["rows"][:, n_q + n_kv:], with_lse=True, window=3000)

        side = T.cuda.Stream()
        with T.cuda.stream(side):
            chain()
        side.synchronize()
        graph = T.cuda.CUDAGraph()
        with T.cuda.graph(graph):
            s["out"] = chain()
        graphs.append((graph, s, chain))
    rng = np.random.default_rng(3)
    for step in range(4):
        for i, (graph, s, chain) in enumerate(graphs):
            q_lens = rng.integers(0, 14, pairs)
            s["doc"].copy_(dev_i32(rng.integers(-1, len(lens), pairs)))
            s["q_lens"].copy_(dev_i32(q_lens))
            s["rows"].copy_(layer_inputs(100 + step * 2 + i, "bf16", n_q, n_kv, d, room))
        for graph, s, _ in graphs:
            graph.replay()
        T.cuda.synchronize()
        for graph, s, chain in graphs:
            n = int(s["tables"].report[0])
            assert n == int(s["q_lens"].sum())
            want = chain(tables=H.PairTables(s["pool"], pairs, room, 313, n_q_heads=n_q))
            T.cuda.synchronize()
            assert T.equal(s["out"][0][:n], want[0][:n]) and T.equal(s["out"][1][:n], want[1][:n])
