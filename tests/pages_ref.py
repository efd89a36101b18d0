"""Plain NumPy forms of the page operators and, in 64 bits, of draft verification."""

import numpy as np


def pages_of(n, page):
    return -(-int(n) // page)


def take(refs, table, places):
    """The lowest free pages to the places (row, column), in order; how many got one, and
    how many are left."""
    free = [int(i) for i in np.flatnonzero(refs == 0)]
    got = min(len(free), len(places))
    for (r, c), p in zip(places, free):
        table[r, c] = p
        refs[p] = 1
    return got, len(free) - got


def resize(refs, page, table, lens, want):
    """refs and table change in place.  Returns lens_out and the free pages left."""
    lens, want = [np.maximum(np.asarray(x, np.int64), 0) for x in (lens, want)]
    places, out = [], []
    for s in range(len(lens)):
        a, b = pages_of(lens[s], page), pages_of(want[s], page)
        for c in range(b, a):
            refs[table[s, c]] -= 1
        places += [(s, c) for c in range(a, b)]
    got, left = take(refs, table, places)
    for s in range(len(lens)):
        a, b = pages_of(lens[s], page), pages_of(want[s], page)
        mine = sum(1 for r, _ in places[:got] if r == s)
        out.append(want[s] if mine == max(b - a, 0) else (a + mine) * page)
    return np.array(out), left


def fork(k, v, refs, page, table, lens, parent, at, out):
    """k, v [L, n_pages, Hkv, page, hd], refs and out (the children's table) change in place.
    Returns lens_out and the free pages left."""
    places, sizes = [], []
    for i, p in enumerate(parent):
        m = 0
        if p >= 0:
            m = max(int(lens[p]), 0)
            if at is not None:
                m = min(m, max(int(at[i]), 0))
        sizes.append(m)
        for c in range(m // page):
            out[i, c] = table[p, c]
            refs[table[p, c]] += 1
        if m % page:
            places.append((i, m // page))
    got, left = take(refs, out, places)
    kk, vv = k.copy(), v.copy()
    for i, c in places[:got]:
        n, src = sizes[i] % page, table[parent[i], c]
        k[:, out[i, c], :, :n] = kk[:, src, :, :n]
        v[:, out[i, c], :, :n] = vv[:, src, :, :n]
    for i, c in places[got:]:
        sizes[i] = c * page
    return np.array(sizes), left


def compact(k, v, page, table, start, keep, n_keep, out):
    """k and v change in place.  Returns lens_out."""
    kk, vv = k.copy(), v.copy()
    lens = []
    for s in range(len(n_keep)):
        a = 0 if start is None else int(start[s])
        n = max(int(n_keep[s]), 0)
        for j in range(n):
            e, d = int(keep[s, j]), a + j
            for x, y in ((k, kk), (v, vv)):
                x[:, out[s, d // page], :, d % page] = y[:, table[s, e // page], :, e % page]
        lens.append(a + n)
    return np.array(lens)


def log_distribution(row, t):
    """Natural logs of the probabilities of logits at temperature t, or None.  (Logs, because a
    token whose probability is below 64 bits' least still has a quotient with another.)"""
    if not 0 <= t <= 2.0 ** 64 or np.isnan(row).any() or (row == np.inf).any() or not (row > -np.inf).any():
        return None
    if t < 2.0 ** -64:
        p = np.full(len(row), -np.inf)
        p[np.argmax(row)] = 0.0
        return p
    with np.errstate(over="ignore"):
        e = (row - row.max()) / t
    return e - np.log(np.exp(e).sum())


def verify(target, draft, drafts, temperature, uniform):
    """target [S, n+1, V] and draft [S, n, V] (or None) float64, drafts int [S, n],
    temperature [S] or None, uniform [S, n+1].  Returns accepted, tokens, logp, and how near
    the closest decision was: |u q / p - 1| over the drafts decided, and the distance of the
    drawn number from the borders of its token, relative to the sums that the token is picked by."""
    S, n1, V = target.shape
    n = n1 - 1
    tokens, logp = np.full((S, n1), -1), np.zeros((S, n1))
    accepted, near, border = np.zeros(S, np.int64), np.inf, np.inf
    for s in range(S):
        t = 1.0 if temperature is None else float(temperature[s])
        greedy = t < 2.0 ** -64
        u = np.clip(np.nan_to_num(uniform[s].astype(np.float64), nan=0.0), 0.0, 1 - 2.0 ** -24)
        for j in range(n1):
            lp, lq = log_distribution(target[s, j], t), None
            if lp is None:
                break
            x = int(drafts[s, j]) if j < n else -1
            if 0 <= x < V:
                if draft is None or greedy:
                    lq = np.full(V, -np.inf)
                    lq[x] = 0.0
                else:
                    lq = log_distribution(draft[s, j], t)
            p = np.exp(lp)
            if lq is None:
                left, size = p, 1.0
            else:
                # u q < p as u q / p < 1 (q = 0: where p > 0; p = 0: never)
                quotient = np.inf if lp[x] == -np.inf else u[j] * np.exp(lq[x] - lp[x]) if lq[x] > -np.inf else 0.0
                if not greedy and np.isfinite(quotient):
                    near = min(near, abs(quotient - 1))
                if quotient < 1:
                    tokens[s, j], logp[s, j] = x, lp[x]
                    accepted[s] += 1
                    continue
                left, size = np.maximum(p - np.exp(lq), 0), 2.0
                if draft is None or greedy:
                    left, size = np.where(np.arange(V) == x, 0, p), 1.0
                if not left.sum() > 0:
                    left, size = p, 1.0
            c = np.cumsum(left)
            goal = u[n] * c[-1]
            tok = int(np.argmax(c > goal))
            border = min(border, (c[tok] - goal) / size, (goal - (c[tok] - left[tok])) / size if goal > 0 else np.inf)
            tokens[s, j], logp[s, j] = tok, lp[tok]
            break
    return accepted, tokens, logp, near, border
