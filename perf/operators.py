"""The operators for models whose layers the caller runs: rotary positions, the tables of a batch of pairs, and the attention
of the pairs' query tokens over their documents' pages.

`run` computes them in plain torch operations, or, with `own` set, with the calls of the library.  Shapes are those of
workloads.MODELS ("tiny": 4 / 4 heads of 64 channels in fp32, 0.5B: 14 / 2 of 64, 8B: 32 / 8 of 128).  The number of documents
and pairs belongs to the case; lengths of an attention case too (its work follows from them), everything else to the seed."""

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 16


# ---- cases ----------------------------------------------------------------------------------------------------------
def _rope(tokens, n_q, n_k, d, rotary, layout, dtype, base, scaling="none", factor=1.0, original=8192, far=4096, **more):
    """`far`: positions are drawn below it.  n_k = 0: one tensor."""
    return dict(op="rope", tokens=tokens, n_q=n_q, n_k=n_k, d=d, rotary=rotary, layout=layout, dtype=dtype, base=base, scaling=scaling,
                factor=factor, original=original, far=far, **more)


def _tables(pairs, docs, doc, query, **more):
    return dict(op="tables", pairs=pairs, docs=docs, doc_lo=doc[0], doc_hi=doc[1], q_lo=query[0], q_hi=query[1], **more)


def _attention(kv, n_q, n_kv, d, pairs, docs, doc, query, cap=0.0, slopes=False, window=0, prefix=False, own_keys=True, lse=False, **more):
    """docs: how many documents the pairs share (0: one of its own for each)."""
    return dict(op="attention", kv=kv, n_q=n_q, n_kv=n_kv, d=d, pairs=pairs, docs=docs, doc_lo=doc[0], doc_hi=doc[1], q_lo=query[0], q_hi=query[1],
                cap=cap, slopes=slopes, window=window, prefix=prefix, own_keys=own_keys, lse=lse, **more)


def listed():
    return [
        # q and k of the shortest request: five candidates, a query of 13 tokens, 0.5B shape
        _rope(65, 14, 2, 64, 64, "half", "bf16", 1.0e6, far=400, name="rope_request_0p5b"),
        # q and k of a batch of 400 pairs at the 8B shape, frequencies stretched by wavelength for a longer context
        _rope(12800, 32, 8, 128, 128, "half", "bf16", 500000.0, "bands", 8.0, 8192, 32768, name="rope_batch_8b"),
        # keys of a document's 24 layers on their way into a pool, fp32, half of each head rotated, neighbouring channels paired, far positions
        _rope(24 * 700, 4, 0, 64, 32, "interleaved", "f32", 10000.0, "ramp", 16.0, 4096, 1 << 20, name="rope_keys_f32"),
        # the tables of one query with 20 candidates: latency
        _tables(20, 60, (100, 512), (32, 32), name="tables_request20"),
        # ... of 256 queries with 100 candidates each over 8192 popular documents
        _tables(25600, 8192, (64, 1024), (8, 64), name="tables_ragged"),
        # a small fp32 model, one query with 8 candidates
        _attention("f32", 4, 4, 64, 8, 0, (128, 128), (16, 16), name="attention_tiny_f32"),
        # one query with 20 candidates, 0.5B shape, scores capped
        _attention("bf16", 14, 2, 64, 20, 0, (512, 512), (32, 32), cap=30.0, name="attention_request20_0p5b"),
        # one token for each of 100 long documents in an 8-bit pool (a second look at its candidates), with the row's log-sum
        _attention("fp8", 32, 8, 128, 100, 0, (2048, 2048), (1, 1), lse=True, name="attention_single_8b_fp8"),
        # 64 short questions about one long document, scores biased by distance
        _attention("bf16", 32, 8, 128, 64, 1, (8192, 8192), (1, 8), slopes=True, name="attention_shared_8b"),
        # one token behind one very long document, 0.5B shape: few rows, a long axis
        _attention("bf16", 14, 2, 64, 1, 0, (32768, 32768), (1, 1), name="attention_one_long_0p5b"),
        # a ragged batch over shared documents, 0.5B shape: a window of 512 tokens, the queries' first tokens seen by all of a query
        _attention("bf16", 14, 2, 64, 2560, 1024, (64, 1024), (8, 64), window=512, prefix=True, name="attention_ragged_0p5b"),
        # the largest: 400 long documents in an 8-bit pool, queries of 64 tokens, 8B shape
        _attention("fp8", 32, 8, 128, 400, 0, (2048, 2048), (64, 64), name="attention_long_8b_fp8"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _span(rng, lo, hi, fixed):
    top = _log_int(rng, lo, hi)
    return (top, top) if rng.random() < fixed else (_log_int(rng, max(1, lo // 2), top), top)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("rope", "tables", "attention", "attention"))
        if op == "rope":
            n_q, n_k, d = rng.choice(((14, 2, 64), (32, 8, 128), (4, 4, 64), (12, 1, 96), (5, 0, 80), (8, 2, 256)))
            rotary = d if rng.random() < 0.6 else 2 * rng.randint(1, d // 2)
            scaling = rng.choice(("none", "linear", "base", "bands", "ramp"))
            factor = 1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0, 32.0))
            if scaling == "base" and rotary <= 2:
                continue
            c = _rope(_log_int(rng, 1, 20000), n_q, n_k, d, rotary, rng.choice(("half", "interleaved")), rng.choice(("bf16", "bf16", "f32")),
                      rng.choice((10000.0, 500000.0, 1.0e6)), scaling, factor, rng.choice((2048, 4096, 8192)), _log_int(rng, 16, 1 << 20))
        elif op == "tables":
            c = _tables(_log_int(rng, 1, 25600), _log_int(rng, 1, 8192), _span(rng, 16, 2048, 0.3), _span(rng, 1, 64, 0.3))
        else:
            kv = rng.choice(("bf16", "bf16", "fp8", "fp8", "f32"))
            n_q, n_kv, d = rng.choice(((4, 4, 64), (8, 2, 32), (6, 1, 80))) if kv == "f32" else rng.choice(((14, 2, 64), (14, 2, 64), (32, 8, 128),
                                                                                                       (32, 8, 128), (8, 1, 128), (12, 4, 96)))
            pairs = _log_int(rng, 1, 40 if kv == "f32" else 640)
            shared = rng.random() < 0.4
            doc = _span(rng, 16, 32768 if shared else 2048, 0.4)
            c = _attention(kv, n_q, n_kv, d, pairs, _log_int(rng, 1, pairs) if shared else 0, doc, _span(rng, 1, 64, 0.4) if rng.random() < 0.7 else (1, 1),
                           cap=rng.choice((0.0, 0.0, 20.0, 50.0)), slopes=rng.random() < 0.3, window=_log_int(rng, 8, 2048) if rng.random() < 0.3 else 0,
                           prefix=rng.random() < 0.3, own_keys=rng.random() < 0.85, lse=rng.random() < 0.3)
            # what the plain form holds: scores in 32 bits, and every pair's keys and values
            keys = c["doc_hi"] + c["q_hi"]
            if 4.0 * pairs * keys * max(c["q_hi"] * n_q, 2 * n_kv * d) > 1.2e10:
                continue
        if _cost(c) <= most:
            return c


# ---- sizes ----------------------------------------------------------------------------------------------------------
def _esz(dtype):
    return {"f32": 4, "bf16": 2, "fp8": 1}[dtype]


def _lengths(c):
    """Documents' lengths, each pair's document, queries' lengths and (prefix) the tokens of a query that all of it sees.  A table's
    rows are 4 bytes whatever they say, so that its lengths follow the seed (prepare); an attention's belong to the case."""
    rng = np.random.default_rng([c["pairs"], c["docs"], c["doc_hi"], c["q_hi"]])
    return _draw_lengths(c, rng)


def _draw_lengths(c, rng):
    n_docs = c["docs"] or c["pairs"]
    doc_lens = rng.integers(c["doc_lo"], c["doc_hi"] + 1, n_docs)
    # popular documents are asked about more often
    pair_doc = (n_docs * rng.random(c["pairs"]) ** 2).astype(np.int64) if c["docs"] else np.arange(c["pairs"])
    q_lens = rng.integers(c["q_lo"], c["q_hi"] + 1, c["pairs"])
    seen = rng.integers(0, q_lens + 1)
    return doc_lens, pair_doc, q_lens, seen


def work(case):
    c = case
    if c["op"] == "rope":
        moved = c["tokens"] * (c["n_q"] + c["n_k"])
        return {"bytes": 2.0 * moved * c["d"] * _esz(c["dtype"]) + 4.0 * c["tokens"], "flops": 3.0 * moved * c["rotary"]}
    if c["op"] == "tables":
        stride = -(-c["doc_hi"] // PAGE)
        tokens = c["pairs"] * c["q_hi"]
        read = 4.0 * (2 * c["pairs"] + 2 * c["docs"] + c["docs"] * (c["doc_lo"] + c["doc_hi"]) / (2 * PAGE))
        return {"bytes": read + 4.0 * (c["pairs"] * (stride + 3) + 2 * tokens), "flops": 0.0}
    doc_lens, pair_doc, q_lens, seen = _lengths(c)
    D, far = doc_lens[pair_doc], c["window"] or 1 << 40
    i = np.arange(c["q_hi"])[None, :]                                    # a pair's tokens, those behind its last masked out
    on = i < q_lens[:, None]
    near = np.maximum(i - far + 1, 0)                                    # the first own key that a token sees
    doc_keys = np.minimum(D[:, None], np.maximum(far - 1 - i, 0))        # a token at D + i sees keys behind D + i - window
    own_keys = np.maximum(np.maximum(i + 1, seen[:, None] if c["prefix"] else 0) - near, 0) if c["own_keys"] else np.zeros_like(i)
    visible = float(((doc_keys + own_keys) * on).sum())
    first = np.minimum(D, far - 1) if c["window"] else D                 # the document keys that some token of the pair sees
    need = np.zeros(len(doc_lens))
    np.maximum.at(need, pair_doc, first)
    tokens, esz = float(q_lens.sum()), _esz("f32" if c["kv"] == "f32" else "bf16")
    nbytes = need.sum() * 2 * c["n_kv"] * c["d"] * _esz(c["kv"]) + tokens * esz * c["d"] * (2 * c["n_q"] + (2 * c["n_kv"] if c["own_keys"] else 0))
    return {"bytes": nbytes + (4.0 * tokens * c["n_q"] if c["lse"] else 0.0), "flops": 4.0 * visible * c["n_q"] * c["d"]}


def _cost(c):
    w = work(c)
    return w["flops"] / 1e15 + w["bytes"] / 4e12


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device=DEV, dtype=dtype)


def _tdt(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _documents(doc_lens, rng):
    """A corpus in a pool: every document's pages, anywhere in it."""
    n_pages = -(-doc_lens // PAGE)
    cu = np.concatenate([[0], np.cumsum(n_pages)])
    return cu, rng.permutation(int(cu[-1])).astype(np.int32)


def _inputs(case, seed):
    c = case
    rng = np.random.default_rng([seed, 7])
    gen = torch.Generator(DEV)
    gen.manual_seed(seed)
    if c["op"] == "rope":
        # rows of a fused projection: q, k and v of a token follow each other
        width = (c["n_q"] + 2 * c["n_k"]) * c["d"]
        rows = torch.randn((c["tokens"], width), generator=gen, device=DEV).to(_tdt(c["dtype"]))
        q = rows[:, :c["n_q"] * c["d"]].unflatten(1, (c["n_q"], c["d"]))
        k = rows[:, c["n_q"] * c["d"]:(c["n_q"] + c["n_k"]) * c["d"]].unflatten(1, (c["n_k"], c["d"])) if c["n_k"] else None
        return dict(case=c, q=q, k=k, positions=_dev(rng.integers(0, c["far"], c["tokens"])))
    doc_lens, pair_doc, q_lens, seen = _draw_lengths(c, rng) if c["op"] == "tables" else _lengths(c)
    page_cu, pages = _documents(doc_lens, rng)
    stride = -(-c["doc_hi"] // PAGE)
    st = dict(case=c, doc_lens=_dev(doc_lens), page_cu=_dev(page_cu), pages=_dev(pages), place=pages, pair_doc=_dev(pair_doc), q_lens=_dev(q_lens), stride=stride,
              pairs=c["pairs"], tokens=c["pairs"] * c["q_hi"] if c["op"] == "tables" else int(q_lens.sum()))
    if c["op"] == "tables":
        return st
    slots, dt = PAGE * len(pages), _tdt(c["kv"])
    st |= dict(q_max=c["q_hi"], doc_max=c["doc_hi"], seen=_dev(seen) if c["prefix"] else None)
    # documents' K and V, page by page in the order of the list; what lies behind a document's end in its last page is zero
    behind = torch.ones(slots, dtype=torch.bool, device=DEV)
    at = np.arange(int(doc_lens.sum())) + np.repeat(page_cu[:-1] * PAGE - np.cumsum(doc_lens) + doc_lens, doc_lens)
    behind[_dev(at, torch.int64)] = False
    shape = (slots, c["n_kv"], c["d"])
    for name in ("k", "v"):
        x = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32 if c["kv"] == "f32" else torch.bfloat16)
        x.masked_fill_(behind[:, None, None], 0.0)
        if c["kv"] == "fp8":
            amax = x.view(len(pages), PAGE, c["n_kv"], c["d"]).abs().amax((1, 3)).float()
            scale = torch.where(amax > 0, amax / 448.0, 1.0)
            codes = (x.view(len(pages), PAGE, c["n_kv"], c["d"]) / scale[:, None, :, None]).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)
            st["doc_" + name], st["scale_" + name] = codes.view(torch.uint8).view(shape), scale
        else:
            st["doc_" + name], st["scale_" + name] = x, None
    draw_rows = lambda heads, size: (torch.randn((st["tokens"], heads, c["d"]), generator=gen, device=DEV) * size).to(dt)  # noqa: E731
    st["q"] = draw_rows(c["n_q"], 3.0)
    st["k"], st["v"] = (draw_rows(c["n_kv"], 1.0), draw_rows(c["n_kv"], 1.0)) if c["own_keys"] else (None, None)
    # slopes fall from head to head by equal factors
    st["slopes"] = torch.exp2(-8.0 * (torch.arange(c["n_q"], device=DEV) + 1) / c["n_q"]) if c["slopes"] else None
    return st


def prepare(case, seed):
    c, st = case, _inputs(case, seed)
    if own:
        from paper_2504_02921_amd import binding as hb
        if c["op"] == "rope":
            st["rope"] = hb.Rope(c["d"], c["base"], rotary_dim=c["rotary"], layout=c["layout"], scaling=c["scaling"], factor=c["factor"],
                                 original_len=c["original"], low=1.0, high=32.0 if c["scaling"] == "ramp" else 4.0)
            return st
        # the corpus of a tables case: pages of one layer of the 0.5B shape that nobody reads
        n_q, n_kv, d, kv = (14, 2, 64, "bf16") if c["op"] == "tables" else (c["n_q"], c["n_kv"], c["d"], c["kv"])
        st["pool"] = hb.KVPool(1, n_kv, d, len(st["place"]), kv, DEV)
        st["tables"] = hb.PairTables(st["pool"], c["pairs"], st["tokens"], st["stride"], n_q_heads=n_q)
        st["docs"] = hb.DocList(st["doc_lens"], st["page_cu"], st["pages"])
        if c["op"] == "attention":
            scales = [st[s][None] for s in ("scale_k", "scale_v")] if c["kv"] == "fp8" else [None, None]
            st["pool"].write(PAGE * len(st["place"]), st["place"], st["doc_k"][None], st["doc_v"][None], *scales)
            st["tables"].build(st["docs"], st["pair_doc"], st["q_lens"])
    return st


# ---- the operators --------------------------------------------------------------------------------------------------
def _frequencies(c):
    """Radians per position of every rotated channel pair, float64, and the factor on the rotated channels."""
    r = c["rotary"]
    base = c["base"] * c["factor"] ** (r / (r - 2.0)) if c["scaling"] == "base" else c["base"]
    f = torch.pow(torch.tensor(base, dtype=torch.float64, device=DEV), torch.arange(r // 2, dtype=torch.float64, device=DEV) * (-2.0 / r))
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "bands":          # by full turns over the original length: 1 and less are stretched, 4 and more are not
        keep = ((c["original"] * f / (2.0 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / c["factor"]
    if c["scaling"] == "ramp":           # the same between 1 and 32 turns, linear in the channel pair's index instead
        index = lambda turns: r * math.log(c["original"] / (2.0 * math.pi * turns)) / (2.0 * math.log(c["base"]))  # noqa: E731
        lo, hi = max(math.floor(index(32.0)), 0), min(math.ceil(index(1.0)), r - 1)
        stretch = ((torch.arange(r // 2, dtype=torch.float64, device=DEV) - lo) / (hi - lo if hi != lo else 0.001)).clamp(0.0, 1.0)
        f = (1.0 - stretch) * f + stretch * f / c["factor"]
    return f, 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "ramp" else 1.0


def _rotated(x, cos, sin, c, work_type):
    r = c["rotary"]
    x = x.to(work_type)
    even, odd = (x[..., 0:r:2], x[..., 1:r:2]) if c["layout"] == "interleaved" else (x[..., :r // 2], x[..., r // 2:r])
    a, b = even * cos - odd * sin, odd * cos + even * sin
    turned = torch.stack((a, b), -1).flatten(-2) if c["layout"] == "interleaved" else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _plain_rope(st):
    c = st["case"]
    f, size = _frequencies(c)
    angle = st["positions"].double()[:, None, None] * f
    cos, sin = (angle.cos() * size).float(), (angle.sin() * size).float()
    q = _rotated(st["q"], cos, sin, c, torch.float32).to(_tdt(c["dtype"]))
    return [q] if st["k"] is None else [q, _rotated(st["k"], cos, sin, c, torch.float32).to(_tdt(c["dtype"]))]


def _plain_tables(st):
    pair_doc, n = st["pair_doc"].long(), st["pairs"]
    q_cu = torch.cat((torch.zeros(1, dtype=torch.int64, device=DEV), st["q_lens"].long().cumsum(0)))
    doc_lens = st["doc_lens"].long()[pair_doc]
    page = torch.arange(st["stride"], device=DEV)[None, :]
    at = (st["page_cu"].long()[pair_doc][:, None] + page).clamp(max=st["pages"].numel() - 1)
    page_table = torch.where(page * PAGE < doc_lens[:, None], st["pages"].long()[at], -1)
    token = torch.arange(st["tokens"], device=DEV)
    pair = torch.searchsorted(q_cu[1:], token, right=True)
    there = pair < n
    safe = pair.clamp(max=n - 1)
    position = torch.where(there, doc_lens[safe] + token - q_cu[safe], -1)
    order = torch.sort(pair_doc, stable=True).indices
    return [t.int() for t in (q_cu, doc_lens, page_table, position, torch.where(there, pair, -1), order)]


def _pairs_rows(st):
    """[pairs][longest query] places of the pairs' tokens, and which of them there are."""
    q_lens = st["q_lens"].long()
    i = torch.arange(st["q_max"], device=DEV)[None, :]
    return (q_lens.cumsum(0) - q_lens)[:, None] + i, i < q_lens[:, None]


def _plain_attention(st):
    c = st["case"]
    g = c["n_q"] // c["n_kv"]
    P, d, D_max, q_max = st["pairs"], c["d"], st["doc_max"], st["q_max"]
    pair_doc = st["pair_doc"].long()
    D = st["doc_lens"].long()[pair_doc]
    rows, on = _pairs_rows(st)
    rows = rows.clamp(max=st["tokens"] - 1)
    j = torch.arange(D_max, device=DEV)[None, :]
    slots = (st["page_cu"].long()[pair_doc][:, None] * PAGE + j).clamp(max=PAGE * st["pages"].numel() - 1)
    there, place = j < D[:, None], j.expand(P, D_max)                    # keys that exist, and their positions

    def documents(name):
        x = st["doc_" + name][slots]
        if c["kv"] == "fp8":
            return x.view(torch.float8_e4m3fn).float() * st["scale_" + name][slots // PAGE][..., None]
        return x.float()

    keys, values = documents("k"), documents("v")
    if c["own_keys"]:
        keys, values = torch.cat((keys, st["k"][rows].float()), 1), torch.cat((values, st["v"][rows].float()), 1)
        there = torch.cat((there, on), 1)
        place = torch.cat((place, D[:, None] + torch.arange(q_max, device=DEV)), 1)
    i = torch.arange(q_max, device=DEV)[None, :]
    ahead = place[:, None, :] - (D[:, None] + i)[:, :, None]             # how far a key lies in front of the query token
    sees = ahead <= 0
    if c["prefix"]:
        sees = sees | (place < (D + st["seen"].long())[:, None])[:, None, :]
    sees = sees & there[:, None, :]
    if c["window"]:
        sees = sees & (ahead > -c["window"])
    q = st["q"][rows].float().unflatten(2, (c["n_kv"], g)).permute(0, 2, 3, 1, 4).reshape(P, c["n_kv"], g * q_max, d)
    s = torch.matmul(q, keys.permute(0, 2, 3, 1).contiguous()).mul_(d ** -0.5).view(P, c["n_q"], q_max, -1)
    if c["cap"]:
        s = s.div_(c["cap"]).tanh_().mul_(c["cap"])
    if st["slopes"] is not None:
        s = s.sub_(st["slopes"][None, :, None, None] * ahead.abs()[:, None].float())
    s = s.masked_fill_(~sees[:, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    values = values.masked_fill(~there[:, :, None, None], 0.0).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p.view(P, c["n_kv"], g * q_max, -1), values).view(P, c["n_q"], q_max, d) / torch.where(total == 0, 1.0, total)
    out = o.permute(0, 2, 1, 3)[on].to(_tdt(c["kv"]))
    return [out, (top + total.log())[..., 0].permute(0, 2, 1)[on]] if c["lse"] else [out]


def run(state):
    c = state["case"]
    if own:
        from paper_2504_02921_amd import binding as hb
        if c["op"] == "rope":
            return state["rope"].apply(state["positions"], *([state["q"]] if state["k"] is None else [state["q"], state["k"]]))
        if c["op"] == "tables":
            t = state["tables"].build(state["docs"], state["pair_doc"], state["q_lens"])
            return [t.q_cu, t.doc_lens, t.page_table, t.tok_pos, t.tok_pair, t.order]
        out = hb.pair_attention(state["pool"], 0, state["tables"], state["q"], state["k"], state["v"], cap=c["cap"], slopes=state["slopes"],
                                window=c["window"], prefix_lens=state["seen"], with_lse=c["lse"])
        return list(out) if c["lse"] else [out]
    return {"rope": _plain_rope, "tables": _plain_tables, "attention": _plain_attention}[c["op"]](state)


# ---- the definitions, in 64 bits --------------------------------------------------------------------------------------
def _exact_frequency(c, i):
    r = c["rotary"]
    base = c["base"] * (c["factor"] ** (r / (r - 2.0)) if c["scaling"] == "base" else 1.0)
    f = base ** (-2.0 * i / r)
    low = f / c["factor"]
    if c["scaling"] == "linear":
        return low
    if c["scaling"] == "bands":
        turns = c["original"] * f / (2.0 * math.pi)
        if turns <= 1.0 or turns >= 4.0:
            return low if turns <= 1.0 else f
        return low + (f - low) * (turns - 1.0) / 3.0
    if c["scaling"] == "ramp":
        pair_of = lambda turns: r * math.log(c["original"] / (2.0 * math.pi * turns)) / (2.0 * math.log(base))  # noqa: E731
        first, last = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), r - 1)
        share = min(max((i - first) / (last - first if last != first else 0.001), 0.0), 1.0)
        return f + (low - f) * share
    return f


def _decoded(codes):
    """E4M3 codes' values: sign, four exponent bits (bias 7; 0: subnormal), three mantissa bits."""
    code = np.arange(256)
    e, m = code >> 3 & 15, (code & 7) / 8.0
    value = np.where(code & 128, -1.0, 1.0) * np.where(e == 0, m * 2.0 ** -6, (1.0 + m) * 2.0 ** (e - 7.0))
    return torch.from_numpy(value).to(DEV)[codes.long()]


def exact(case, seed):
    c = case
    if c["op"] == "tables":
        return None
    st = _inputs(case, seed)
    if c["op"] == "rope":
        r, size = c["rotary"], 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "ramp" else 1.0
        f = torch.tensor([_exact_frequency(c, i) for i in range(r // 2)], dtype=torch.float64, device=DEV)
        turn = torch.polar(torch.full_like(f, size), torch.zeros_like(f)) * torch.exp(1j * (st["positions"].double()[:, None] * f))
        result = []
        for x in (st["q"], st["k"]):
            if x is None:
                continue
            y = x.double().clone()
            first, second = (slice(0, r, 2), slice(1, r, 2)) if c["layout"] == "interleaved" else (slice(0, r // 2), slice(r // 2, r))
            z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn[:, None, :]
            y[..., first], y[..., second] = z.real, z.imag
            result.append(y)
        return result
    doc_lens, pair_doc, q_lens, seen = _lengths(c)
    g, first_slot = c["n_q"] // c["n_kv"], PAGE * np.concatenate([[0], np.cumsum(-(-doc_lens // PAGE))])
    out, logs, t0 = [], [], 0
    for p in range(c["pairs"]):                                          # pair by pair, all of its heads together
        D, n, doc = int(doc_lens[pair_doc[p]]), int(q_lens[p]), int(pair_doc[p])
        span, page = slice(int(first_slot[doc]), int(first_slot[doc]) + D), torch.arange(int(first_slot[doc]), int(first_slot[doc]) + D, device=DEV) // PAGE
        kv = []
        for name in ("k", "v"):
            x = st["doc_" + name][span]
            x = _decoded(x) * st["scale_" + name].double()[page][..., None] if c["kv"] == "fp8" else x.double()
            if c["own_keys"]:
                x = torch.cat((x, st[name][t0:t0 + n].double()))
            kv.append(x.transpose(0, 1).repeat_interleave(g, 0))         # [n_q][keys][d]
        at = torch.arange(D + (n if c["own_keys"] else 0), device=DEV)[None, :]
        me = D + torch.arange(n, device=DEV)[:, None]
        logits = st["q"][t0:t0 + n].double().transpose(0, 1) @ kv[0].transpose(1, 2).contiguous() / math.sqrt(c["d"])
        if c["cap"]:
            logits = c["cap"] * torch.tanh(logits / c["cap"])
        if st["slopes"] is not None:
            logits = logits - st["slopes"].double()[:, None, None] * (me - at).abs()
        hidden = at > me
        if c["prefix"]:
            hidden = hidden & (at >= D + int(seen[p]))
        if c["window"]:
            hidden = hidden | (me - at >= c["window"])
        logits = logits.masked_fill(hidden, -math.inf)
        log = torch.logsumexp(logits, -1)
        weight = torch.exp(logits - torch.where(log == -math.inf, 0.0, log)[..., None])
        out.append((weight @ kv[1]).transpose(0, 1))
        logs.append(log.transpose(0, 1))
        t0 += n
    return [torch.cat(out), torch.cat(logs)] if c["lse"] else [torch.cat(out)]

