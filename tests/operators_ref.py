"""64-bit references of the operators for models whose layers the caller runs (rotary positions, tables of a batch of pairs, attention over
document pages), and bounds on what rounding may add."""

import numpy as np

PAGE = 16
U32, U16, UBF = 2.0 ** -24, 2.0 ** -11, 2.0 ** -8      # half a step of fp32, half, bf16 relative to the value


def rope(x, pos, freqs, layout, amplitude=1.0, inverse=False):
    """x [T][heads][d], pos [T] -> rotated, and the sum of the magnitudes that went into every output."""
    x = np.asarray(x, np.float64)
    r = 2 * len(freqs)
    ang = np.asarray(pos, np.float64)[:, None, None] * np.asarray(freqs)[None, None, :] * (-1.0 if inverse else 1.0)
    c, s = np.cos(ang) * amplitude, np.sin(ang) * amplitude
    i = np.arange(r // 2)
    first, second = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + r // 2)
    y, size = x.copy(), np.zeros_like(x)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size[..., first] = size[..., second] = (np.abs(a) + np.abs(b)) * amplitude
    return y, size


def tables(doc_lens, page_cu, pages, num_pages, pair_doc, query_lens, max_tokens, pt_stride):
    """What hr_pair_tables_build fills: a dict of arrays, and the report's bits."""
    n, n_docs = len(pair_doc), len(doc_lens)
    bits = 0
    cu, t = np.zeros(n + 1, np.int32), 0
    for p, q in enumerate(query_lens):
        if q < 0 or t + max(q, 0) > max_tokens:
            bits |= 2
        t = min(t + max(int(q), 0), max_tokens)
        cu[p + 1] = t
    lens, table = np.zeros(n, np.int32), np.full((n, pt_stride), -1, np.int32)
    keys = np.zeros(n, np.int64)
    for p, doc in enumerate(pair_doc):
        if not 0 <= doc < n_docs:
            bits |= 0 if doc == -1 else 1
            continue
        keys[p] = doc + 1
        lo = min(max(page_cu[doc], 0), len(pages))
        hi = min(max(page_cu[doc + 1], lo), len(pages))
        lens[p] = min(max(doc_lens[doc], 0), min(hi - lo, pt_stride) * PAGE)
        bits |= 4 if lens[p] != doc_lens[doc] else 0
        k = -(-int(lens[p]) // PAGE)
        ids = np.asarray(pages[lo:lo + k])
        bad = (ids < 0) | (ids >= num_pages)
        bits |= 8 if bad.any() else 0
        table[p, :k] = np.where(bad, -1, ids)
    pos, pair = np.full(max_tokens, -1, np.int32), np.full(max_tokens, -1, np.int32)
    for p in range(n):
        pos[cu[p]:cu[p + 1]] = lens[p] + np.arange(cu[p + 1] - cu[p])
        pair[cu[p]:cu[p + 1]] = p
    return dict(q_cu=cu, doc_lens=lens, page_table=table, tok_pos=pos, tok_pair=pair, order=np.argsort(keys, kind="stable").astype(np.int32),
                report=np.array([cu[-1], len(set(keys.tolist())), bits, 0], np.int32))


def attention(q, k, v, docs, pair_doc, q_lens, scale=None, cap=0.0, slopes=None, window=0, prefix=None, pool="bf16"):
    """q [T][n_q][d]; k, v [T][n_kv][d] or None; docs: list of (K, V) [D][n_kv][d].  Returns out, log-sum, and a bound on the error of each.

    The bound, per output: one rounding to the output's type; weights off by their rounding to half (16-bit and fp8 pools: U16 of each, and
    2^-25 where they are below half's normal range: the largest weight is at least 1) and by the score's error; fp32 sums of n terms.
    A score is off by the sum over d of fp32 products and by the roundings of its scaling, cap, bias and exponential."""
    f = np.float64
    T, n_q, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    half = pool != "f32"
    out, log = np.zeros((T, n_q, d), f), np.full((T, n_q), -np.inf)
    tol, tol_log = np.zeros((T, n_q, d), f), np.zeros((T, n_q), f)
    t0 = 0
    for p, n in enumerate(q_lens):
        n, doc = int(n), int(pair_doc[p])
        K, V = [], []
        n_kv = (k if k is not None else docs[0][0]).shape[1]
        D = 0
        if doc >= 0:
            K, V, D = [docs[doc][0].astype(f)], [docs[doc][1].astype(f)], docs[doc][0].shape[0]
        if k is not None:
            K, V = K + [k[t0:t0 + n].astype(f)], V + [v[t0:t0 + n].astype(f)]
        K = np.concatenate(K) if K else np.zeros((0, n_kv, d))
        V = np.concatenate(V) if V else np.zeros((0, n_kv, d))
        j, i = np.arange(len(K))[None, :], D + np.arange(n)[:, None]
        sees = j <= i
        if prefix is not None:
            sees |= j < D + min(max(int(prefix[p]), 0), n)
        if window:
            sees &= i - j < window
        for a in range(n_q if n else 0):
            h = a // (n_q // n_kv)
            qa = q[t0:t0 + n, a].astype(f)
            with np.errstate(all="ignore"):
                s = scale * (qa @ np.where(np.isfinite(K[:, h]), K[:, h], 0.0).T) if len(K) else np.zeros((n, 0))
                size = abs(scale) * (np.abs(qa) @ np.abs(np.where(np.isfinite(K[:, h]), K[:, h], 0.0)).T) if len(K) else np.zeros((n, 0))
            if cap:
                s = cap * np.tanh(s / cap)
            if slopes is not None:
                s = s - float(slopes[a]) * np.abs(i - j)
            s = np.where(sees, s, -np.inf)
            if not len(K):
                continue
            m = s.max(1, keepdims=True)
            m0 = np.where(m == -np.inf, 0.0, m)
            w = np.exp(s - m0)
            l = w.sum(1, keepdims=True)
            l1 = np.where(l == 0, 1.0, l)
            Vh = V[:, h]
            odd = ~np.isfinite(Vh)
            o = (w @ np.where(odd, 0.0, Vh)) / l1
            for y, x in zip(*np.nonzero(odd)):                       # a value that is not finite counts where its key is seen
                with np.errstate(invalid="ignore"):
                    o[sees[:, y], x] += Vh[y, x]
            mag = (w @ np.abs(np.where(odd, 0.0, Vh))) / l1
            out[t0:t0 + n, a] = o
            with np.errstate(divide="ignore"):
                log[t0:t0 + n, a] = np.where(l[:, 0] > 0, m0[:, 0] + np.log(l[:, 0]), -np.inf)
            ds = U32 * ((d + 8) * np.where(sees, size, 0.0).max(1) + 16 * np.abs(np.where(sees, s, 0.0)).max(1) + 8 * cap)[:, None]
            terms = len(K) * U32
            tol[t0:t0 + n, a] = (UBF if half else U32) * np.abs(np.where(np.isfinite(o), o, 0.0)) + (2 * ds + 2 * terms + 4 * U32 + (U16 if half else 0.0)) * mag
            if half:
                tol[t0:t0 + n, a] += len(K) * 2.0 ** -25 * np.abs(np.where(odd, 0.0, Vh)).max() if len(K) else 0.0
            tol_log[t0:t0 + n, a] = 2 * ds[:, 0] + terms + 4 * U32 * (1 + np.abs(np.where(l[:, 0] > 0, log[t0:t0 + n, a], 0.0)))
        t0 += n
    return out, log, tol, tol_log
