"""Plain NumPy forms, in 64 bits, of the paged-cache and beam-search operators."""

import numpy as np

F32_HALF = 2.0 ** -24   # half a step of float32, relative
BF16_HALF = 2.0 ** -8   # half a step of bfloat16, relative


def rope(x, pos, theta):
    """x [..., hd] rotated to pos (broadcast over the leading axes of x)."""
    hd = x.shape[-1]
    f = float(theta) ** (-2.0 * np.arange(hd // 2) / hd)
    a = np.asarray(pos, np.float64)[..., None] * f
    c, s = np.cos(a), np.sin(a)
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)


def entries(pool, row, n):
    """[Hkv, n, hd]: the first n entries behind a table row."""
    _, Hkv, page, hd = pool.shape
    used = -(-n // page)
    return pool[np.asarray(row[:used], np.int64)].transpose(1, 0, 2, 3).reshape(Hkv, used * page, hd)[:, :n]


def attention(k, v, q, table, lens, groups=None, ptable=None, plens=None, weighted=None):
    """q [S, n_q, Hq, hd]; groups: cu_seqs.  Returns out and lse2 (NaN rows for
    padding sequences).  weighted: when a dict, receives sum p |v| and the largest
    sum |q_d k_d| / sqrt(hd) of a row, for error bounds."""
    S, n_q, Hq, hd = q.shape
    Hkv = k.shape[1]
    out, lse = np.full(q.shape, np.nan), np.full(q.shape[:3], np.nan)
    spread, size = np.zeros(q.shape), 0.0
    for s in range(S):
        g = None
        if groups is not None:
            live = [i for i in range(len(groups) - 1) if groups[i] <= s < groups[i + 1]]
            if not live:
                continue
            g = live[0]
        for j in range(n_q):
            own = max(0, lens[s] - n_q + j + 1)
            kk, vv = entries(k, table[s], own), entries(v, table[s], own)
            if g is not None:
                kk = np.concatenate([entries(k, ptable[g], plens[g]), kk], axis=1)
                vv = np.concatenate([entries(v, ptable[g], plens[g]), vv], axis=1)
            for h in range(Hq):
                kh, vh, qh = kk[h // (Hq // Hkv)], vv[h // (Hq // Hkv)], q[s, j, h]
                if kh.shape[0] == 0:
                    out[s, j, h], lse[s, j, h] = 0.0, -np.inf
                    continue
                w = kh @ qh / np.sqrt(hd)
                m = w.max()
                p = np.exp(w - m)
                out[s, j, h] = p @ vh / p.sum()
                lse[s, j, h] = (m + np.log(p.sum())) / np.log(2.0)
                spread[s, j, h] = p @ np.abs(vh) / p.sum()
                size = max(size, float((np.abs(kh) @ np.abs(qh)).max()) / np.sqrt(hd))
    if weighted is not None:
        weighted.update(spread=spread, size=size)
    return out, lse


def attention_tol(out, weighted, keys, hd, bf16):
    """Bounds of |error| of out and lse2.  A float32 product sum of hd terms is off by
    at most hd 2^-24 of the sum of its terms' sizes, which moves a probability by that
    much, relatively; the sum of `keys` of them by keys 2^-24 more, the exponential by
    2^-22, the bf16 pair that carries P by 2^-17.  Numerator and denominator move: twice.
    Then one rounding of the result."""
    eps = hd * F32_HALF * weighted["size"] + keys * F32_HALF + 2.0 ** -22 + (2.0 ** -17 if bf16 else 0.0)
    tol = 2 * eps * weighted["spread"] + (BF16_HALF if bf16 else F32_HALF) * np.abs(out) * (1 + 2 * eps) + 1e-30
    return tol, (2 * eps + 2.0 ** -22) / np.log(2.0)


def select(logits, scores, done, eos, K):
    """logits [B, W, V] float32, scores [B, W], done [B, W] or None.  Returns scores
    (64 bits), parent, token, done of the K best, in the operator's order, and the
    smallest gap between two different totals of different beams around them."""
    B, W, V = logits.shape
    out, gap = [], np.inf
    for b in range(B):
        tot, par, tok, lg = [], [], [], []
        for w in range(W):
            x = logits[b, w].astype(np.float64)
            s = 0.0 if scores is None else float(scores[b, w])
            if done is not None and done[b, w]:
                x = np.full(V, -np.inf)
                x[eos] = 0.0
                lse = 0.0
            elif np.isnan(x).any() or (x == np.inf).any():
                x = np.where(np.isnan(x), -np.inf, x)
                lse = np.nan
            elif (x == -np.inf).all():
                lse = 0.0
            else:
                lse = x.max() + np.log(np.exp(x - x.max()).sum())
            with np.errstate(invalid="ignore"):
                t = s + (x - lse)
            top = np.lexsort((np.arange(V), -x))[:K]
            tot += list(t[top])
            par += [w] * len(top)
            tok += list(top)
            lg += list(x[top])
        tot, par, tok, lg = np.array(tot), np.array(par), np.array(tok), np.array(lg)
        key = np.where(np.isnan(tot), -np.inf, tot)
        order = np.lexsort((tok, -lg, par, -key, np.isnan(tot)))
        near = order[:K + 1]
        for a, c in zip(near[:-1], near[1:]):
            if par[a] != par[c] and np.isfinite(tot[a]) and np.isfinite(tot[c]) and tot[a] != tot[c]:
                gap = min(gap, tot[a] - tot[c])
        order = order[:K]
        ended = np.array([tok[i] == eos or (done is not None and done[b, par[i]]) for i in order])
        out.append((tot[order], par[order], tok[order], ended))
    return tuple(np.stack([o[i] for o in out]) for i in range(4)) + (gap,)


def reorder(k, v, parent, table, lens, fresh, cols):
    """k, v [L, n_pages, Hkv, page, hd] (changed in place).  Returns table_out (-9 where
    nothing is written) and lens_out."""
    B, K = parent.shape
    W, page = table.shape[0] // B, k.shape[3]
    out, out_lens = np.full((B * K, cols), -9), np.zeros(B * K, np.int64)
    kk, vv = k.copy(), v.copy()
    for b in range(B):
        seen = set()
        for j in range(K):
            s, o = b * W + parent[b, j], b * K + j
            whole, part = divmod(int(lens[s]), page)
            out[o, :whole] = table[s, :whole]
            out_lens[o] = lens[s]
            if part and parent[b, j] not in seen:
                out[o, whole] = table[s, whole]
            else:
                if whole < cols:
                    out[o, whole] = fresh[o]
                if part:
                    k[:, fresh[o], :, :part] = kk[:, table[s, whole], :, :part]
                    v[:, fresh[o], :, :part] = vv[:, table[s, whole], :, :part]
            seen.add(parent[b, j])
    return out, out_lens
