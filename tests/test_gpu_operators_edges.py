"""The operators for models whose layers the caller runs, where sizes, masks and values come to an end: odd heads, large caps, rows of NaN, outputs
over inputs, tiles in pieces.  References and bounds are those of operators_ref.py."""

import numpy as np
import pytest

import operators_ref as R
from oracle import fp8 as ofp8
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


# ---- attention ----------------------------------------------------------------------------------------------------------
def check_cap(b, cap, **a):
    """As Batch.check, with a bound that does not grow with the cap.  A capped score is no larger than the score and no farther from its own value than
    the score is, so the bound of the scores without a cap holds (it has 16 half steps of a score for what is done to it; the cap takes 17 at most, of a
    sum of magnitudes that has d + 8 and is no smaller than the score); it is taken out of the bound of the log-sum without a cap.  The rest is
    operators_ref's: weights, sums of as many terms as there are keys, one rounding of the output."""
    n = b.tokens
    out, lse = b.run(cap=cap, **a)
    x = [to64(t)[:n] for t in (b.q, b.k, b.v)]
    a = dict(a, slopes=None if a.get("slopes") is None else to64(a["slopes"]))
    ref = lambda v, docs, cap: R.attention(x[0], x[1], v, docs, b.pair_doc, b.q_lens, cap=cap, pool=b.kv, **a)      # noqa: E731
    want, log, _, _ = ref(x[2], b.docs, cap)
    _, log0, _, tol0 = ref(x[2], b.docs, 0.0)
    sizes = ref(np.abs(x[2]), [(k, np.abs(v)) for k, v in b.docs], cap)[0]
    keys = np.repeat([b.docs[doc][0].shape[0] + m for doc, m in zip(b.pair_doc, b.q_lens)], b.q_lens)[:, None]
    scores = (tol0 - keys * R.U32 - 4 * R.U32 * (1 + np.abs(log0))) / 2
    half = b.kv != "f32"
    tol = (R.UBF if half else R.U32) * np.abs(want) + (2 * scores + 2 * keys * R.U32 + 4 * R.U32 + (R.U16 if half else 0.0))[..., None] * sizes
    if half:
        tol += (keys * 2.0 ** -25)[..., None] * max(np.abs(v).max() for v in [x[2]] + [v for _, v in b.docs])
    tol_log = 2 * scores + keys * R.U32 + 4 * R.U32 * (1 + np.abs(log))
    err, err_log = np.abs(to64(out)[:n] - want), np.abs(to64(lse)[:n] - log)
    assert np.all(err <= tol), f"cap {cap}: out, max err / bound {np.max(err / tol):.2f}"
    assert np.all(err_log <= tol_log), f"cap {cap}: log-sum, max err / bound {np.max(err_log / tol_log):.2f}"


@pytest.mark.parametrize("kv,n_q,n_kv,d", [("bf16", 14, 2, 64), ("bf16", 12, 4, 96), ("bf16", 8, 1, 128), ("fp8", 6, 2, 64), ("fp8", 6, 2, 96), ("fp8", 32, 8, 128),
                                           ("bf16", 5, 1, 80), ("f32", 4, 4, 64)])
@pytest.mark.parametrize("pairs,doc,query", [(2, 1000, 3), (70, 200, 37)])
def test_a_cap_does_not_cost_the_score_its_digits(kv, n_q, n_kv, d, pairs, doc, query):
    """From caps that the scores reach to those that change none of them, in blocks, pieces and tiles."""
    T = torch()
    b = Batch(kv, n_q, n_kv, d, np.random.default_rng(pairs).integers(doc // 2, doc + 1, pairs), np.arange(pairs), np.full(pairs, query), seed=5, layers=1, layer=0)
    for cap in (0.5, 20.0, 64.0, 1e3, 1e5, 1e8, 1e18):
        check_cap(b, cap)
    check_cap(b, 1e6, slopes=T.full((n_q,), 0.01, device=DEV), window=doc // 3, scale=-0.1)


@pytest.mark.parametrize("kv,n_q,n_kv,d", [("bf16", 14, 2, 64), ("fp8", 8, 2, 128), ("bf16", 6, 2, 96), ("bf16", 5, 1, 80), ("f32", 4, 4, 64)])
@pytest.mark.parametrize("pairs,doc,query", [(3, 60, 5), (1, 6000, 2), (2, 900, 20), (90, 100, 40)])
def test_a_row_of_nan_has_neither_a_value_nor_a_log_sum(kv, n_q, n_kv, d, pairs, doc, query):
    """Scores that are all NaN, in blocks, in few and many pieces and in tiles: the row's output and log-sum are NaN, the other rows' are as they were."""
    T = torch()
    b = Batch(kv, n_q, n_kv, d, [doc] * pairs, np.arange(pairs), [query] * pairs, seed=11, layers=1, layer=0)
    out, lse = b.run()
    q = b.q.clone()
    q[1, 0], q[-1, n_q - 1, 3] = float("nan"), float("nan")
    hit = T.zeros((b.tokens, n_q), dtype=T.bool, device=DEV)
    hit[1, 0] = hit[-1, n_q - 1] = True
    for own in (True, False):
        out, lse = b.run(own)
        bad, bad_lse = b.run(own, q=q)
        assert bool(T.isnan(bad[hit]).all()) and bool(T.isnan(bad_lse[hit]).all())
        assert T.equal(bad[~hit], out[~hit]) and T.equal(bad_lse[~hit], lse[~hit])
    # a key that the rows behind it see beside others
    k = b.k.clone()
    k[query - 1, 0] = float("nan")
    bad, bad_lse = b.run(k=k)
    out, lse = b.run()
    g = n_q // n_kv
    assert bool(T.isnan(bad[query - 1, :g]).all()) and bool(T.isnan(bad_lse[query - 1, :g]).all())
    assert T.equal(bad[:query - 1], out[:query - 1]) and T.equal(bad_lse[:query - 1], lse[:query - 1]) and T.equal(bad[query:], out[query:])


def test_tables_that_were_not_built_are_refused():
    T, H = torch(), hb()
    b = Batch("bf16", 4, 2, 64, [20], [0], [3])
    t = H.PairTables(b.pool, 1, 3, 2, n_q_heads=4)
    with pytest.raises(H.HrError):
        H.pair_attention(b.pool, 0, t, b.q, b.k, b.v)
    t.build(b.list, dev_i32([0]), dev_i32([3]))
    assert T.equal(H.pair_attention(b.pool, b.layer, t, b.q, b.k, b.v), b.run()[0])


def test_gradients_are_refused_and_not_dropped():
    T, H = torch(), hb()
    b = Batch("bf16", 4, 2, 64, [20], [0], [3])
    rope = H.Rope(64)
    want, want_q = b.run()[0], rope.apply(0, b.q)[0]
    for name in ("q", "k", "v"):
        x = getattr(b, name).clone().requires_grad_()
        with pytest.raises(H.HrError, match="no_grad"):
            b.run(**{name: x})
        with T.no_grad():
            assert T.equal(b.run(**{name: x})[0], want)
    x = b.q.clone().requires_grad_()
    for call in (lambda: rope.apply(0, x), lambda: rope.apply(0, b.q, x), lambda: rope.apply(0, b.q, out=[x]), lambda: b.run(out=x),
                 lambda: b.run(slopes=T.zeros(4, device=DEV, requires_grad=True))):
        with pytest.raises(H.HrError, match="no_grad"):
            call()
    with T.no_grad():
        assert T.equal(rope.apply(0, x)[0], want_q)
    assert T.equal(rope.apply(0, x.detach())[0], want_q)


def test_inputs_on_another_stream_outlive_the_callers_hold_on_them():
    """What a call on a busy stream still has to read is not given out again: nothing is written, only asked for."""
    T, H = torch(), hb()
    pairs = 300000
    b = Batch("bf16", 4, 2, 64, [20], [0], [4000])
    t, side = H.PairTables(b.pool, pairs, 16, 2, n_q_heads=4), T.cuda.Stream()
    rope = H.Rope(64)

    def build():
        doc, lens = (T.zeros(pairs, dtype=T.int32, device=DEV) for _ in range(2))
        call = lambda: t.build(b.list, doc, lens, stream=side)                                      # noqa: E731
        return call, [doc, lens]

    def turn():
        x, pos = T.zeros((300000, 2, 64), dtype=T.bfloat16, device=DEV), T.zeros(300000, dtype=T.int32, device=DEV)
        return (lambda: rope.apply(pos, x, stream=side)), [x, pos]

    def attend():
        q, k, v = b.q.clone(), b.k.clone(), b.v.clone()
        return (lambda: b.run(q=q, k=k, v=v, stream=side)), [q, k, v]

    for make in (build, turn, attend):
        T.cuda.synchronize()
        call, held = make()
        T.cuda.synchronize()
        with T.cuda.stream(side):
            T.cuda._sleep(100_000_000)
        result = call()
        places = {x.data_ptr() for x in held}
        like = [(x.shape, x.dtype) for x in held]
        busy = not side.query()
        del call, held
        fresh = [T.empty(shape, dtype=dtype, device=DEV) for shape, dtype in like]
        assert busy and not places & {x.data_ptr() for x in fresh}, make.__name__
        T.cuda.synchronize()
        del result


# ---- tiles ---------------------------------------------------------------------------------------------------------------
def choice(b):
    """Whether the device takes tiles for a batch, and into how many pieces it cuts their keys: the rule of pair_choice, on the counts of the built list."""
    blocks, tiles = (int(x) * b.n_kv for x in b.tables.sched[2:4].tolist())
    rows = b.tables.max_tokens * b.n_q
    most = max(1, round(b.tables.workspace_bytes / (rows * (8 + 4 * b.d))))
    is_tiles = blocks > (512 if b.d == 64 else 256) and 2 * blocks > 3 * tiles
    return is_tiles, min(max(512 // max(tiles if is_tiles else blocks, 1), 1), most)


TILE_SHAPES = [("bf16", 14, 2, 64), ("fp8", 14, 2, 64), ("bf16", 12, 4, 96), ("fp8", 12, 4, 96), ("bf16", 16, 2, 128), ("fp8", 8, 1, 128)]


def tile_batch(kv, n_q, n_kv, d, cut, spare=0, seed=21):
    """Pairs of a long document, of a short one, of none, with queries of no token to many, in no order; or the same behind documents that are not cut."""
    rng = np.random.default_rng(seed)
    pairs, rows = 40, 1600 * n_kv * 7 // n_q if d == 64 else 1200 * 8 * n_kv // (n_q * min(n_kv, 2))
    docs = [2101, 45, 31] if cut else [500, 45, 333]
    doc = rng.choice([0, 0, 0, 0, 1, 2, -1], pairs) if cut else rng.choice([0, 1, 2, -1], pairs)
    lens = rng.multinomial(rows, rng.dirichlet(np.ones(pairs) * 3.0))
    lens[[3, 17]] = [0, 1]
    b = Batch(kv, n_q, n_kv, d, docs, doc, lens, seed=seed, spare=spare)
    is_tiles, pieces = choice(b)
    assert is_tiles and (pieces > 1) == cut, (is_tiles, pieces)
    return b


@pytest.mark.parametrize("kv,n_q,n_kv,d", TILE_SHAPES)
@pytest.mark.parametrize("cut", [False, True])
def test_tiles_whole_and_in_pieces(kv, n_q, n_kv, d, cut):
    T = torch()
    b = tile_batch(kv, n_q, n_kv, d, cut)
    pairs = len(b.q_lens)
    prefix = dev_i32(np.where(np.arange(pairs) % 3 == 0, 0, b.q_lens * (np.arange(pairs) % 4) // 2) - 1)      # none, in the query, past its end
    slopes = T.full((n_q,), 0.01, device=DEV)
    b.check(what="plain")
    b.check(prefix_lens=prefix, what="prefix")
    b.check(window=300, prefix_lens=prefix, what="prefix and window")
    b.check(own=False, window=40, what="pieces that see nothing, rows that see nothing")
    b.check(window=9, what="window inside the queries")
    b.check(cap=20.0, slopes=slopes, window=450, prefix_lens=prefix, scale=-0.1, what="all")


@pytest.mark.parametrize("kv,n_q,n_kv,d", TILE_SHAPES)
@pytest.mark.parametrize("cut", [False, True])
def test_tiles_leave_alone_what_is_not_theirs(kv, n_q, n_kv, d, cut):
    """Values that are not finite where nobody looks, packed rows one element off, outputs between others, rows behind the last token."""
    T = torch()
    b = tile_batch(kv, n_q, n_kv, d, cut, spare=5, seed=22)
    cu = np.concatenate([[0], np.cumsum(b.q_lens)])
    long = [p for p in range(len(b.q_lens)) if b.q_lens[p] >= 12][:6]
    prefix = dev_i32(np.minimum(b.q_lens // 3, 4))
    for a in (dict(), dict(window=200), dict(prefix_lens=prefix, window=100), dict(prefix_lens=prefix)):
        out, lse = b.run(**a)
        q, k, v = (t.clone() for t in (b.q, b.k, b.v))
        for t in (q, k, v):
            t[b.tokens:] = float("nan")
        hit = np.zeros(b.tokens, bool)
        for i, p in enumerate(long):                                        # a key late in a pair's query: the tokens from it on see it
            at = cu[p] + b.q_lens[p] - 1 - i
            (v if i % 2 else k)[at] = float("nan") if i < 3 else float("inf")
            hit[at:cu[p + 1]] = True
        keep = T.from_numpy(~hit).to(DEV)
        bad, bad_lse = b.run(q=q, k=k, v=v, **a)
        assert T.equal(bad[:b.tokens][keep], out[:b.tokens][keep]) and T.equal(bad_lse[:b.tokens][keep], lse[:b.tokens][keep])
        assert not bool(T.isfinite(bad[:b.tokens][~keep]).all(-1).any())
        n = b.q.shape[0]
        flat = T.zeros(n * (n_q + 2 * n_kv) * d + 1, dtype=b.q.dtype, device=DEV)
        rows = flat[1:].view(n, n_q + 2 * n_kv, d)
        rows[:, :n_q], rows[:, n_q:n_q + n_kv], rows[:, n_q + n_kv:] = b.q, b.k, b.v
        rows[b.tokens:] = float("nan")
        wide = T.full((n_q + 2, n, d + 4), 3.0, dtype=b.q.dtype, device=DEV)
        into = wide[1:1 + n_q, :, :d].transpose(0, 1)
        got, got_lse = b.run(q=rows[:, :n_q], k=rows[:, n_q:n_q + n_kv], v=rows[:, n_q + n_kv:], out=into, **a)
        assert T.equal(got[:b.tokens], out[:b.tokens]) and T.equal(got_lse[:b.tokens], lse[:b.tokens])
        assert bool((into[b.tokens:] == 3.0).all()) and bool((wide[0] == 3.0).all()) and bool((wide[n_q + 1] == 3.0).all()) and bool((wide[:, :, d:] == 3.0).all())


@pytest.mark.parametrize("kv,n_q,n_kv,d", TILE_SHAPES + [("bf16", 5, 1, 80), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("stride", [1, 60])
def test_a_long_query_without_a_document_attends_to_itself(kv, n_q, n_kv, d, stride):
    """A prompt's own causal attention; with room for long documents, so that pieces begin among the own keys."""
    b = Batch(kv, n_q, n_kv, d, [10], [-1, 0, -1], [1400, 33, 90], seed=23, stride=stride)
    if kv != "f32" and d in (64, 96, 128):                                  # the kernels that know tiles
        assert choice(b)[0] and (choice(b)[1] > 1) == (stride == 60), choice(b)
    b.check(what="causal")
    b.check(window=100, what="window")
    b.check(prefix_lens=dev_i32([50, 33, 0]), what="prefix")


# ---- sizes at their ends --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_pairs", [5, 300, 6000])
def test_tables_without_a_single_document(n_pairs):
    H = hb()
    rng = np.random.default_rng(n_pairs)
    pool = H.KVPool(1, 2, 16, 1, "bf16", DEV)
    pair_doc, q_lens = rng.choice([-1, -1, 0, 7], n_pairs), rng.integers(0, 5, n_pairs)
    none = np.zeros(0, np.int64)
    t = H.PairTables(pool, n_pairs, int(q_lens.sum()), 0, n_q_heads=14)
    t.build(H.DocList(dev_i32(none), dev_i32([0]), dev_i32(none)), dev_i32(pair_doc), dev_i32(q_lens))
    for name, w in R.tables(none, np.zeros(1, np.int64), none, 1, pair_doc, q_lens, int(q_lens.sum()), 0).items():
        np.testing.assert_array_equal(getattr(t, name).cpu().numpy(), w, err_msg=name)


@pytest.mark.parametrize("kv,d", [("bf16", 128), ("fp8", 128), ("bf16", 96), ("bf16", 80), ("f32", 128)])
@pytest.mark.parametrize("pairs", [3, 90])
def test_attention_of_pages_and_rows_past_32_bits(kv, d, pairs):
    """Pages at the end of a pool of more than 4 GiB, rows of q, k, v and out that far apart: the bits of the same call close together."""
    T, H = torch(), hb()
    n_q, n_kv, D, query = 8, 8, 70, 12
    rng = np.random.default_rng(pairs)
    page = 2 * R.PAGE * d * n_kv * {"bf16": 2, "fp8": 1, "f32": 4}[kv]
    n_pages = (5 << 30) // page
    k, v = (rng.standard_normal((1, D, n_kv, d)) for _ in range(2))
    if kv == "fp8":
        (kc, ks), (vc, vs) = ofp8.quantize_doc_kv(k), ofp8.quantize_doc_kv(v)
        given = [T.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in (kc, vc, ks.astype(np.float32), vs.astype(np.float32))]
    else:
        given = [T.from_numpy(x).to(dtype_of(kv)).to(DEV) for x in (k, v)]
    tokens = pairs * query
    gen = T.Generator().manual_seed(1)
    rows = [T.randn((tokens, n, d), generator=gen).to(dtype_of(kv)).to(DEV) for n in (n_q, n_kv, n_kv)]
    results = []
    for pages in (5, n_pages):
        pool = H.KVPool(1, n_kv, d, pages, kv, DEV)
        ids = np.arange(pages - 5, pages, dtype=np.int32)
        pool.write(D, ids, *given)
        t = H.PairTables(pool, pairs, tokens, 5, n_q_heads=n_q).build(H.DocList(dev_i32([D]), dev_i32([0, 5]), dev_i32(ids)), dev_i32(np.zeros(pairs)), dev_i32(np.full(pairs, query)))
        apart = rows
        if pages == n_pages:
            step = ((5 << 30) // (4 if kv == "f32" else 2) // tokens + d) // 8 * 8
            assert step * (tokens - 1) * (4 if kv == "f32" else 2) > 1 << 32 and step >= (n_q + 2 * n_kv) * d
            room = T.zeros(step * tokens, dtype=rows[0].dtype, device=DEV).view(tokens, step)
            cut, at = [], 0
            for x in rows:
                cut.append(room[:, at:at + x.shape[1] * d].unflatten(1, (x.shape[1], d)))
                cut[-1].copy_(x)
                at += x.shape[1] * d
            apart = cut
            out = T.zeros_like(room)[:, :n_q * d].unflatten(1, (n_q, d))
        else:
            out = T.zeros_like(rows[0])
        results.append(H.pair_attention(pool, 0, t, *apart, out=out, with_lse=True))
        T.cuda.synchronize()
    assert T.equal(results[0][0], results[1][0]) and T.equal(results[0][1], results[1][1]) and bool(T.isfinite(results[0][0]).all())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_of_rows_past_32_bits(layout):
    T, H = torch(), hb()
    tokens, heads, d = (1 << 18) + 3, 64, 128
    x = T.zeros((tokens, heads, d), dtype=T.bfloat16, device=DEV)
    assert x.numel() > 1 << 31
    some = T.randn((5, heads, d), generator=T.Generator().manual_seed(1)).to(T.bfloat16).to(DEV)
    x[:2], x[-3:] = some[:2], some[2:]
    rope = H.Rope(d, 10000.0, layout=layout)
    want, = rope.apply(dev_i32([0, 1, tokens - 3, tokens - 2, tokens - 1]), some)
    y, = rope.apply(0, x)
    assert T.equal(y[:2], want[:2]) and T.equal(y[-3:], want[2:])
    rope.apply(0, x, out=[x])
    assert T.equal(y, x)


def test_calls_on_a_second_stream_of_a_recording():
    """Tables, rotary positions and attention on a stream that a recording forks to; its positions and keys are temporaries that are let go of."""
    T, H = torch(), hb()
    b = Batch("bf16", 14, 2, 64, [900, 40], [0, 1, 0], [5, 9, 1], seed=31)
    rope = H.Rope(64)
    doc, lens, rows = dev_i32(b.pair_doc), dev_i32(b.q_lens), [b.q.clone(), b.k.clone(), b.v.clone()]
    t = H.PairTables(b.pool, 3, b.tokens, 57, n_q_heads=14)
    side, other, graph = T.cuda.Stream(), T.cuda.Stream(), T.cuda.CUDAGraph()

    def chain(stream):
        t.build(b.list, doc, lens, stream=stream)
        q, k = rope.apply(t.tok_pos, rows[0], rows[1], stream=stream)
        return H.pair_attention(b.pool, b.layer, t, q, k, rows[2], with_lse=True, stream=stream)

    T.cuda.synchronize()
    with T.cuda.stream(side):
        chain(None)
    side.synchronize()
    with T.cuda.graph(graph):
        now = T.cuda.current_stream()
        other.wait_stream(now)
        out = chain(other)
        now.wait_stream(other)
    gen = T.Generator().manual_seed(2)
    for _ in range(4):
        for x in rows:
            x.copy_(T.randn(x.shape, generator=gen).to(x.dtype))
        q_lens = np.random.default_rng(3).permutation(b.q_lens)
        lens.copy_(dev_i32(q_lens))
        graph.replay()
        T.cuda.synchronize()
        got = [x.clone() for x in out]
        want = chain(None)
        T.cuda.synchronize()
        assert T.equal(got[0], want[0]) and T.equal(got[1], want[1])
