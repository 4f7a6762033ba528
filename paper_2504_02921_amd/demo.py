"""End-to-end walk through the library on one GPU: prefill a few documents into a paged pool, score every (query,
document) pair with only the query tokens run through the layers, pick each query's best candidates, run one layer operator by operator
(norms, projections in 8 bits, rotary positions, attention over the same pool), move a document to pinned host memory and back (16-bit records, then 4-bit ones).  Random weights and token ids; run as `python -m paper_2504_02921_amd.demo`."""

import numpy as np


def layer_of_the_callers(pool, cfg, docs, doc_pages, query_lens, window: int = 64):
    """One layer as a caller runs it whose model hr_rerank_score does not cover: norms, projections in 8 bits, rotary positions, tables built on the device,
    attention with a window over the documents' pages (layer 0), a gated feed-forward.  Every document gets one query.  Returns the attention's largest
    difference from plain torch operations, and the projections' distance from fp32 ones with the weights as they were, relative to what those give."""
    import torch

    from . import binding as hb

    dev, n, tokens = pool.mem.device, len(docs), int(sum(query_lens))
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(dev)      # noqa: E731
    n_pages = [len(p) for p in doc_pages]
    listed = hb.DocList(i32([len(d) for d in docs]), i32(np.concatenate([[0], np.cumsum(n_pages)])), i32(np.concatenate(doc_pages)))
    tables = hb.PairTables(pool, n, tokens, max(n_pages), n_q_heads=cfg.n_q_heads)
    tables.build(listed, i32(np.arange(n)), i32(query_lens))
    gen = torch.Generator(device=dev).manual_seed(0)
    normal = lambda *shape: torch.randn(shape, generator=gen, device=dev)                  # noqa: E731
    heads = cfg.n_q_heads * cfg.head_dim
    plain = [normal(rows, cols) * cols ** -0.5 for rows, cols in ((cfg.qkv_out, cfg.hidden), (cfg.hidden, heads), (2 * cfg.ffn, cfg.hidden), (cfg.hidden, cfg.ffn))]
    qkv_w, out_w, up_w, down_w = (hb.block_quantize(w, hb.BLOCK_COLS) for w in plain)
    gains = 1 + 0.1 * normal(2, cfg.hidden)
    x = normal(tokens, cfg.hidden).bfloat16()

    rows = hb.block_matmul(hb.rms_norm(x, gains[0], eps=cfg.rms_eps, out=None, block8=True)[2], qkv_w)
    q, k, v = (part.unflatten(1, (-1, cfg.head_dim)) for part in rows.split([heads, cfg.n_kv_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim], 1))
    q, k = hb.Rope(cfg.head_dim, cfg.rope_base).apply(tables.tok_pos, q, k)
    out = hb.pair_attention(pool, 0, tables, q, k, v, window=window)
    x2 = hb.block_matmul(hb.block_quantize(out.flatten(1)), out_w, add=x)
    up = hb.block_matmul(hb.rms_norm(x2, gains[1], eps=cfg.rms_eps, out=None, block8=True)[2], up_w, gate="silu", block8=True)
    y = hb.block_matmul(up, down_w, add=x2)

    normed = lambda s, gain: s * (s.square().mean(-1, keepdim=True) + cfg.rms_eps).rsqrt() * gain      # noqa: E731
    s = x.float() + out.flatten(1).float() @ plain[1].t()
    gate, lin = (normed(s, gains[1]) @ plain[2].t()).chunk(2, 1)
    s = s + (gate * torch.sigmoid(gate) * lin) @ plain[3].t()
    away = max(float((a.float() - b).norm() / b.norm()) for a, b in ((rows, normed(x.float(), gains[0]) @ plain[0].t()), (y, s)))

    gap, t0 = 0.0, 0
    for doc, pages, m in zip(docs, doc_pages, query_lens):
        kd, vd = (x[0].float() for x in pool.read(len(doc), pages))
        keys, values = (torch.cat([d, own[t0:t0 + m].float()]).repeat_interleave(cfg.group, 1) for d, own in ((kd, k), (vd, v)))
        s = torch.einsum("ihd,jhd->hij", q[t0:t0 + m].float(), keys) * cfg.head_dim ** -0.5
        behind = (len(doc) + torch.arange(m, device=dev))[:, None] - torch.arange(len(doc) + m, device=dev)[None]
        s = s.masked_fill((behind < 0) | (behind >= window), float("-inf"))
        gap = max(gap, float((torch.einsum("hij,jhd->ihd", s.softmax(-1), values) - out[t0:t0 + m].float()).abs().max()))
        t0 += m
    return gap, away


def main(n_queries: int = 3, n_docs: int = 6, doc_len: int = 200, query_len: int = 24, top_k: int = 2, verbose: bool = True):
    import torch

    from . import binding as hb
    from . import workloads as wlmod

    dev = "cuda:0"
    cfg = wlmod.ModelCfg("demo", 4, 512, 8, 2, 64, 1408, 4096, 1e6, 1e-6, dtype="bf16")     # a small Qwen2-shaped decoder
    weights = wlmod.SeededWeights(cfg, seed=1, std=0.05)
    model = hb.Model(cfg, weights, dev)
    rng = np.random.default_rng(0)

    # stage one: every document's K/V of every layer, computed once and kept in pool pages
    pages_per_doc = (doc_len + hb.PAGE_TOKENS - 1) // hb.PAGE_TOKENS
    pool = hb.KVPool(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, n_docs * pages_per_doc + 8, "bf16", dev)
    docs = [rng.integers(0, cfg.vocab, doc_len).astype(np.int32) for _ in range(n_docs)]
    doc_pages = [pool.alloc(pages_per_doc) for _ in range(n_docs)]
    model.doc_prefill(pool, docs, doc_pages)

    # stage two: each query against every document; only the query tokens go through the layers
    queries = [rng.integers(0, cfg.vocab, query_len).astype(np.int32) for _ in range(n_queries)]
    page_table = np.stack([doc_pages[d] for _ in range(n_queries) for d in range(n_docs)]).astype(np.int32)
    doc_lens = np.full(n_queries * n_docs, doc_len, np.int32)
    q_tokens = np.concatenate([queries[q] for q in range(n_queries) for _ in range(n_docs)])
    q_lens = np.full(n_queries * n_docs, query_len, np.int32)
    scores = model.score(pool, page_table, doc_lens, q_tokens, q_lens)
    seg = np.arange(0, n_queries * n_docs + 1, n_docs)
    best = hb.rerank_topk(scores, seg, top_k)
    torch.cuda.synchronize()

    # the same scores without reuse: the full [document ; query] sequence per pair
    full = model.score_full([docs[d] for _ in range(n_queries) for d in range(n_docs)],
                            [queries[q] for q in range(n_queries) for _ in range(n_docs)])
    torch.cuda.synchronize()
    gap = float((scores - full).abs().max())

    layer_gap, layer_away = layer_of_the_callers(pool, cfg, docs, doc_pages, [query_len] * n_docs)

    # host tier: evict document 0 to pinned host memory, free its pages, bring it back at other pages
    rec = torch.empty(pages_per_doc * pool.page_record_bytes, dtype=torch.uint8, pin_memory=True)
    pool.pages_out(doc_pages[0], rec)
    torch.cuda.synchronize()
    pool.free(doc_pages[0])
    spare = pool.alloc(8)                      # the lowest free pages: the spare ones are not among them any more
    new_pages = pool.alloc(pages_per_doc)
    pool.free(spare)
    pool.pages_in(new_pages, rec)
    page_table2 = page_table.copy()
    page_table2[0::n_docs] = new_pages
    again = model.score(pool, page_table2, doc_lens, q_tokens, q_lens)
    torch.cuda.synchronize()
    same = bool(torch.equal(scores, again))

    # the same through 4-bit records: a third of the bytes over the bus, scores change by the quantisation
    rec4 = torch.empty(pages_per_doc * pool.page_record4_bytes, dtype=torch.uint8, pin_memory=True)
    pool.pages_out4(new_pages, rec4)
    torch.cuda.synchronize()
    pool.free(new_pages)
    pool.pages_in4(new_pages, rec4)
    lossy = model.score(pool, page_table2, doc_lens, q_tokens, q_lens)
    torch.cuda.synchronize()
    change4 = float((lossy - scores).abs().max())

    if verbose:
        for q in range(n_queries):
            print(f"query {q}: best documents {best[q].tolist()}  scores {[round(float(scores[q * n_docs + int(d)]), 4) for d in best[q]]}")
        print(f"max |reuse - full recompute| = {gap:.2e}; scores after the host-tier round trip identical: {same}; "
              f"after a round trip of one document in 4 bits they move by at most {change4:.2e}")
        print(f"a layer of the caller's own: windowed attention over the pool differs from plain operations by at most {layer_gap:.2e}, projections in 8 bits "
              f"from fp32 ones by {100 * layer_away:.1f} %")
    model.close()
    pool.close()
    return scores.cpu().numpy(), best.cpu().numpy(), gap, same


if __name__ == "__main__":
    main()
