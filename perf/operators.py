"""Several continuations of one prompt over paged caches, as measurable cases.

Four operators that a generation step uses one after the other:

* ``append``     a step's (or a prompt's) keys and values into a paged cache, keys
                 rotated to their positions on the way, and the rotated queries.
* ``attention``  the step's queries over a prompt that all sequences of a group
                 share and over each sequence's own pages.
* ``select``     the best continuations over a batch element's beams and vocabulary.
* ``reorder``    page tables that follow the chosen beams, with the last, partly
                 filled page copied where two beams continue the same parent.

Cache pages are ``[page, KV head, entry, dim]``; a table row lists a sequence's
pages in order, -1 past its last one.  Layer sizes are those of the repository's
1B, 8B and float32 configurations (``inputs.py``) or generic ones.  Lengths of a
ragged batch follow from the case alone, every value from the seed.

Where ``own`` is false, ``run`` computes the same in elementary torch operations:
32 bits, 64 for the angles of far positions and for the totals that continuations
are ranked by.
"""

from __future__ import annotations

import math
import random

import torch

own = False

LOG2E = 1.4426950408889634
EOS = 2

HEADS_1B = dict(Hq=32, Hkv=8, hd=64, theta=500000.0, dtype="bf16")
HEADS_8B = dict(Hq=32, Hkv=8, hd=128, theta=500000.0, dtype="bf16")
HEADS_F32 = dict(Hq=4, Hkv=4, hd=32, theta=10000.0, dtype="f32")


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # One generated token for each of 8 sequences of the 1B shape, products in
        # float32 as a decode step leaves them: the smallest call, launch latency.
        dict(name="append_token_1b_s8", op="append", S=8, rows=1, ctx=130, page=16, ragged=False, wide=True, **HEADS_1B),
        # Prompts of up to 2048 tokens of the 8B shape going into the cache.
        dict(name="append_prompt_8b", op="append", S=6, rows=2048, ctx=0, page=64, ragged=True, wide=False, **HEADS_8B),
        # Beam search on one short prompt, 1B shape: latency of a layer's attention.
        dict(name="attend_beams_1b", op="attention", S=4, G=1, prefix=99, suffix=21, nq=1, page=16, ragged=False,
             **HEADS_1B),
        # Eight prompts of the 8B shape pruned to about 1200 rows, 4 beams each.
        dict(name="attend_beams_8b", op="attention", S=32, G=8, prefix=1204, suffix=160, nq=1, page=32, ragged=True,
             **HEADS_8B),
        # One long document, 64 samples of an answer to it.
        dict(name="attend_document_8b", op="attention", S=64, G=1, prefix=32000, suffix=600, nq=1, page=64, ragged=True,
             **HEADS_8B),
        # No shared prompt: single tokens over long caches of their own.
        dict(name="attend_own_8b", op="attention", S=48, G=0, prefix=0, suffix=4001, nq=1, page=16, ragged=True,
             **HEADS_8B),
        # Four drafted tokens per sequence checked together, groups of uneven size.
        dict(name="attend_drafts_1b", op="attention", S=24, G=3, prefix=2047, suffix=301, nq=4, page=16, ragged=True,
             **HEADS_1B),
        # The float32 heads, drafts of three tokens.
        dict(name="attend_f32", op="attention", S=12, G=4, prefix=413, suffix=77, nq=3, page=16, ragged=True, **HEADS_F32),
        # Four beams of one prompt over the whole vocabulary, twice as many kept.
        dict(name="select_b1_w4", op="select", B=1, W=4, V=128256, K=8, pad=0, masked=False, done=False),
        # A serving batch: 24 prompts of 8 beams, banned tokens, finished beams, an
        # odd vocabulary in padded rows.
        dict(name="select_b24_w8", op="select", B=24, W=8, V=128003, K=8, pad=13, masked=True, done=True),
        # Beams of one prompt of the 1B shape, all layers.
        dict(name="reorder_1b_w4", op="reorder", L=16, B=1, W=4, K=4, len=141, kept=2, page=16, ragged=False, **HEADS_1B),
        # The 8B shape, 16 prompts of 8 beams, pages nearly full.
        dict(name="reorder_8b_w8", op="reorder", L=32, B=16, W=8, K=8, len=190, kept=4, page=64, ragged=True, **HEADS_8B),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    if rng.random() < 0.2:
        hd, dtype = rng.choice([32, 64, 128]), "f32"
    else:
        hd, dtype = rng.choice([64, 128]), "bf16"
    Hkv, per = rng.choice([(8, 4), (8, 4), (4, 2), (2, 8), (1, 5), (5, 3), (12, 1)])
    return dict(Hq=Hkv * per, Hkv=Hkv, hd=hd, theta=rng.choice([10000.0, 500000.0]), dtype=dtype)


def draw(rng: random.Random):
    while True:
        case = _drawn(rng)
        w = work(case)
        if w["bytes"] <= 500e6 and w["flops"] <= 30e9:  # within the largest listed ones
            return case


def _drawn(rng):
    op = rng.choice(["append", "attention", "attention", "select", "reorder"])
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        rows = _log_int(rng, 1, 1500) if rng.random() < 0.6 else 1
        return dict(op=op, S=_log_int(rng, 1, 64) if rows < 100 else rng.randint(1, 6), rows=rows, ctx=_log_int(rng, 1, 3000),
                    page=page, ragged=rng.random() < 0.5, wide=rng.random() < 0.5, **_heads(rng))
    if op == "attention":
        h = _heads(rng)
        S = _log_int(rng, 1, 64)
        G = rng.choice([0, 1, rng.randint(1, S)])
        most = 24000 if h["dtype"] == "bf16" else 3000
        prefix = min(_log_int(rng, 1, most), 100000 // G) if G else 0
        suffix = min(_log_int(rng, 1, most // 4), 90000 // S)
        return dict(op=op, S=S, G=G, prefix=prefix, suffix=suffix, nq=rng.choice([1, 1, 1, 2, 5]), page=page,
                    ragged=rng.random() < 0.7, **h)
    if op == "select":
        W = rng.randint(1, 12)
        B, V = _log_int(rng, 1, 24 * 8 // W), _log_int(rng, 900, 128256)
        return dict(op=op, B=B, W=W, V=V, K=rng.choice([W, 2 * W, rng.randint(1, 24)]), pad=rng.randint(0, 9),
                    masked=rng.random() < 0.5, done=rng.random() < 0.5)
    W, K = rng.randint(1, 8), rng.randint(1, 8)
    h = _heads(rng)
    return dict(op=op, L=_log_int(rng, 1, 32), B=_log_int(rng, 1, 16), W=W, K=K, len=_log_int(rng, 1, 600),
                kept=rng.randint(1, min(W, K)), page=page, ragged=rng.random() < 0.5, **h)


# ------------------------------------------------------------------ sizes that follow from a case

def _spread(case, n, most, salt):
    """n lengths: all `most`, or for a ragged case between half of it and it."""
    if not case["ragged"]:
        return [most] * n
    r = random.Random(1000003 * n + 101 * most + salt)
    return [r.randint(max(1, most - most // 2), most) if most else 0 for _ in range(n)]


def _group_ends(case):
    """[0, end of group 0, ..., S]: groups in order, at least one sequence each."""
    S, G = case["S"], case["G"]
    if not G:
        return [0]
    if not case["ragged"]:
        return [g * S // G for g in range(G + 1)]
    r = random.Random(7919 * S + G)
    return [0] + sorted(r.sample(range(1, S), G - 1)) + [S]


def _append_sizes(case):
    n = _spread(case, case["S"], case["rows"], 1)
    ctx = _spread(case, case["S"], case["ctx"], 2)
    return n, [a + b for a, b in zip(n, ctx)]


def _attention_sizes(case):
    lens = [max(x, case["nq"]) for x in _spread(case, case["S"], case["suffix"], 3)]
    return lens, _spread(case, case["G"], case["prefix"], 4), _group_ends(case)


def _reorder_lens(case):
    return _spread(case, case["B"], case["len"], 5)


def _esz(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    op = case["op"]
    if op == "select":
        rows = case["B"] * case["W"]
        return dict(bytes=rows * case["V"] * 4 + rows * 5 + case["B"] * case["K"] * 13, flops=3 * rows * case["V"])
    Hkv, hd, e = case["Hkv"], case["hd"], _esz(case)
    if op == "append":
        n, lens = _append_sizes(case)
        T, width = sum(n), (case["Hq"] + 2 * Hkv) * hd
        e_in = 4 if case["wide"] else e
        tables = sum(-(-b // case["page"]) - (b - a) // case["page"] for a, b in zip(n, lens))
        return dict(bytes=T * width * (e_in + e) + 4 * (T + tables + 2 * case["S"] + 1), flops=3 * T * (case["Hq"] + Hkv) * hd)
    if op == "attention":
        lens, plens, ends = _attention_sizes(case)
        nq, Hq = case["nq"], case["Hq"]
        rows = case["S"] * nq * Hq
        keys = sum(lens) + sum(plens)
        seen = nq * sum(lens) - case["S"] * nq * (nq - 1) // 2
        seen += nq * sum((b - a) * p for a, b, p in zip(ends, ends[1:], plens))
        return dict(bytes=2 * keys * Hkv * hd * e + 2 * rows * hd * e + 4 * rows + 4 * (keys // case["page"] + case["S"]),
                    flops=4 * seen * Hq * hd)
    lens = _reorder_lens(case)
    entry = 2 * Hkv * hd * e * case["L"]
    moved = (case["K"] - case["kept"]) * sum(n % case["page"] for n in lens) * entry
    tables = 4 * case["K"] * sum(2 * (n // case["page"] + 1) + 4 for n in lens)
    return dict(bytes=2 * moved + tables, flops=0)


# ------------------------------------------------------------------ inputs

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _tables(lens, page, free, cols):
    """One row of page numbers per sequence, taken from the list of free pages."""
    rows = []
    for n in lens:
        used = -(-n // page)
        rows.append([free.pop() for _ in range(used)] + [-1] * (cols - used))
    return _ints(rows)


def _free(n_pages, seed):
    free = list(range(n_pages))
    random.Random(seed).shuffle(free)
    return free


def _pool(g, n_pages, case, *layers):
    size = (*layers, n_pages, case["Hkv"], case["page"], case["hd"])
    return [torch.randn(size, generator=g, device="cuda", dtype=_type(case)) for _ in range(2)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return dict(append=_prepare_append, attention=_prepare_attention, select=_prepare_select,
                reorder=_prepare_reorder)[case["op"]](case, seed, g)


def _prepare_append(case, seed, g):
    n, lens = _append_sizes(case)
    page, Hq, Hkv, hd = case["page"], case["Hq"], case["Hkv"], case["hd"]
    T, cols = sum(n), max(-(-x // page) for x in lens) + 1
    n_pages = sum(-(-x // page) for x in lens) + 3
    k, v = _pool(g, n_pages, case)
    width = (Hq + 2 * Hkv) * hd
    qkv = torch.randn(T, width, generator=g, device="cuda", dtype=torch.float32)
    # positions of a pruned prompt have gaps, and reach further than its entries
    pos = torch.cumsum(torch.randint(1, 9, (T,), generator=g, device="cuda"), 0).to(torch.int32)
    ends = [0]
    for x in n:
        ends.append(ends[-1] + x)
    return dict(case=case, k=k, v=v, qkv=qkv if case["wide"] else qkv.to(_type(case)), pos=pos, T=T, cols=cols,
                cu=None if case["rows"] == 1 else _ints(ends), cu_all=_ints(ends), lens=_ints(lens),
                table=_tables(lens, page, _free(n_pages, seed), cols),
                q_out=torch.empty(T, Hq, hd, device="cuda", dtype=_type(case)))


def _prepare_attention(case, seed, g):
    lens, plens, ends = _attention_sizes(case)
    page, S, nq, Hq, hd = case["page"], case["S"], case["nq"], case["Hq"], case["hd"]
    cols = max(-(-x // page) for x in lens) + 1
    pcols = max([-(-x // page) for x in plens], default=0)
    n_pages = sum(-(-x // page) for x in lens + plens) + 2
    k, v = _pool(g, n_pages, case)
    free = _free(n_pages, seed)
    q = (1.5 * torch.randn(S, nq, Hq, hd, generator=g, device="cuda")).to(_type(case))
    return dict(case=case, k=k, v=v, q=q, lens=_ints(lens), table=_tables(lens, page, free, cols), cols=cols, pcols=pcols,
                ends=_ints(ends), most=max([b - a for a, b in zip(ends, ends[1:])], default=0),
                plens=_ints(plens) if case["G"] else None,
                ptable=_tables(plens, page, free, pcols) if case["G"] else None,
                out=torch.empty(S, nq, Hq, hd, device="cuda", dtype=_type(case)),
                lse=torch.empty(S, nq, Hq, device="cuda", dtype=torch.float32))


def _prepare_select(case, seed, g):
    B, W, V, K = case["B"], case["W"], case["V"], case["K"]
    rows = 3.0 * torch.randn(B * W, V + case["pad"], generator=g, device="cuda", dtype=torch.float32)
    if case["masked"]:  # tokens that a grammar or a repetition rule bans
        rows[torch.rand(rows.shape, generator=g, device="cuda") < 0.3] = -math.inf
    scores = -20.0 * torch.rand(B, W, generator=g, device="cuda", dtype=torch.float32)
    done = torch.rand(B, W, generator=g, device="cuda") < (0.2 if case["done"] else 0.0)
    return dict(case=case, logits=rows, scores=scores, done=done.to(torch.uint8),
                scores_out=torch.empty(B, K, device="cuda", dtype=torch.float32),
                parent=torch.empty(B, K, device="cuda", dtype=torch.int32),
                token=torch.empty(B, K, device="cuda", dtype=torch.int32),
                done_out=torch.empty(B, K, device="cuda", dtype=torch.uint8))


def _prepare_reorder(case, seed, g):
    B, W, K, page = case["B"], case["W"], case["K"], case["page"]
    lens = [n for n in _reorder_lens(case) for _ in range(W)]
    cols = max(lens) // page + 2
    # whole pages of a batch element are shared by its beams, the partial one is each beam's own
    n_pages = sum(n // page for n in _reorder_lens(case)) + B * (W + K) + 1
    free = _free(n_pages, seed)
    rows, r = [], random.Random(seed + 1)
    for n in _reorder_lens(case):
        whole = [free.pop() for _ in range(n // page)]
        rows += [whole + [free.pop()] + [-1] * (cols - len(whole) - 1) for _ in range(W)]
    parent = []
    for _ in range(B):
        chosen = r.sample(range(W), case["kept"])
        row = chosen + [r.choice(chosen) for _ in range(K - case["kept"])]
        r.shuffle(row)
        parent.append(row)
    k, v = _pool(g, n_pages, case, case["L"])
    return dict(case=case, k=k, v=v, parent=_ints(parent), table=_ints(rows), cols=cols, lens=_ints(lens),
                fresh=_ints([free.pop() for _ in range(B * K)]),
                table_out=torch.full((B * K, cols), -1, dtype=torch.int32, device="cuda"),
                lens_out=torch.zeros(B * K, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------ one pass

def run(state):
    return dict(append=_run_append, attention=_run_attention, select=_run_select,
                reorder=_run_reorder)[state["case"]["op"]](state)


def _library():
    from paper_2509_01190_gb300 import zsaa
    return zsaa


def _run_append(st):
    c = st["case"]
    if own:
        z = _library()
        if "pages" not in st:
            st["pages"] = z.make_pages(st["k"], st["v"])
        z.zsaa_op_paged_append(st["pages"], st["qkv"], st["qkv"].shape[1], z.ZSAA_F32 if st["qkv"].dtype == torch.float32 else z.ZSAA_BF16,
                               st["T"], c["Hq"], st["pos"], c["theta"], st["cu"], c["S"], st["table"], st["cols"], st["lens"],
                               st["q_out"])
        return st["q_out"], st["k"], st["v"]
    Hq, Hkv, hd, page = c["Hq"], c["Hkv"], c["hd"], c["page"]
    rows = torch.arange(st["T"], device="cuda")
    seq = torch.searchsorted(st["cu_all"][1:], rows, right=True)
    entry = (st["lens"][seq] - st["cu_all"][seq + 1]).long() + rows
    pages = st["table"][seq, entry // page].long()
    x = st["qkv"].float().reshape(st["T"], Hq + 2 * Hkv, hd)
    half = hd // 2
    freq = c["theta"] ** (-2.0 * torch.arange(half, device="cuda", dtype=torch.float64) / hd)
    angle = st["pos"].double()[:, None] * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = x[:, :Hq + Hkv, :half], x[:, :Hq + Hkv, half:]
    turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2).to(_type(c))
    st["k"][pages, :, entry % page] = turned[:, Hq:]
    st["v"][pages, :, entry % page] = x[:, Hq + Hkv:].to(_type(c))
    return turned[:, :Hq], st["k"], st["v"]


def _gathered(pool, table):
    """[rows, KV head, entry, dim] in 32 bits of a table's pages (hidden entries are of no account)."""
    n, cols = table.shape
    x = pool[table.long()].float()
    return x.transpose(1, 2).reshape(n, pool.shape[1], cols * pool.shape[2], pool.shape[3])


def _run_attention(st):
    c = st["case"]
    S, G, nq, Hq, Hkv, hd = c["S"], c["G"], c["nq"], c["Hq"], c["Hkv"], c["hd"]
    if own:
        z = _library()
        if "pages" not in st:
            st["pages"] = z.make_pages(st["k"], st["v"])
            n = z.zsaa_op_paged_attention_workspace(st["pages"], S, nq, Hq, G, st["cols"], st["pcols"])
            st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        z.zsaa_op_paged_attention(st["pages"], st["q"], S, nq, Hq, st["table"], st["cols"], st["lens"],
                                  st["ends"] if G else None, G, st["ptable"], st["pcols"], st["plens"], st["out"], st["lse"],
                                  st["ws"], st["ws"].numel())
        return st["out"], st["lse"]
    per = Hq // Hkv
    q = st["q"].float().reshape(S, nq, Hkv, per, hd).transpose(1, 2).reshape(S, Hkv, nq * per, hd)
    i = torch.arange(st["cols"] * c["page"], device="cuda")
    j = torch.arange(nq * per, device="cuda") // per
    seen = i <= st["lens"][:, None, None] - nq + j[:, None]
    s = torch.matmul(q, _gathered(st["k"], st["table"]).transpose(2, 3)) / math.sqrt(hd)
    s = torch.where(seen[:, None], s, -math.inf)
    top = s.amax(3, keepdim=True)
    if G:
        seat = torch.arange(st["most"], device="cuda")
        rows = torch.clamp(st["ends"][:-1, None] + seat, max=S - 1).long()
        n = torch.arange(S, device="cuda")
        group = torch.searchsorted(st["ends"][1:], n, right=True)
        at = n - st["ends"][group]
        qg = q[rows].transpose(1, 2).reshape(G, Hkv, st["most"] * nq * per, hd)
        sp = torch.matmul(qg, _gathered(st["k"], st["ptable"]).transpose(2, 3)) / math.sqrt(hd)
        ip = torch.arange(st["pcols"] * c["page"], device="cuda")
        sp = torch.where(ip < st["plens"][:, None, None, None], sp, -math.inf)
        per_seq = lambda t: t.reshape(G, Hkv, st["most"], nq * per, -1).transpose(1, 2)[group, at]  # noqa: E731
        top = torch.maximum(top, per_seq(sp.amax(3, keepdim=True)))
        top_g = top[rows].transpose(1, 2).reshape(G, Hkv, -1, 1)
        ep = torch.exp(sp - top_g)
        total_p, sum_p = per_seq(ep.sum(3, keepdim=True)), per_seq(torch.matmul(ep, _gathered(st["v"], st["ptable"])))
    e = torch.exp(s - top)
    total, weighted = e.sum(3, keepdim=True), torch.matmul(e, _gathered(st["v"], st["table"]))
    if G:
        total, weighted = total + total_p, weighted + sum_p
    back = lambda t: t.reshape(S, Hkv, nq, per, -1).transpose(1, 2).reshape(S, nq, Hq, -1)  # noqa: E731
    return back(weighted / total).to(_type(c)), back(LOG2E * (top + torch.log(total)))[..., 0]


def _run_select(st):
    c = st["case"]
    B, W, V, K = c["B"], c["W"], c["V"], c["K"]
    if own:
        z = _library()
        if "ws" not in st:
            st["ws"] = torch.empty(z.zsaa_op_beam_select_workspace(B, W, V, K), dtype=torch.uint8, device="cuda")
        z.zsaa_op_beam_select(st["logits"], V + c["pad"], B, W, V, st["scores"], st["done"], EOS, K, st["scores_out"],
                              st["parent"], st["token"], st["done_out"], st["ws"], st["ws"].numel())
        return st["scores_out"], st["parent"], st["token"], st["done_out"]
    done = st["done"].reshape(B * W, 1).bool()
    only = torch.where(torch.arange(V, device="cuda") == EOS, 0.0, -math.inf)
    x = torch.where(done, only, st["logits"][:, :V])
    best, token = torch.sort(x, dim=1, descending=True, stable=True)
    best, token = best[:, :K].double(), token[:, :K]
    lse = best[:, :1] + torch.log(torch.exp(x.double() - best[:, :1]).sum(1, keepdim=True))
    total = (st["scores"].reshape(B * W, 1).double() + (best - lse)).reshape(B, -1)
    total, at = torch.sort(total, dim=1, descending=True, stable=True)
    total, at = total[:, :K], at[:, :K]
    n = best.shape[1]
    parent, token = at // n, token.reshape(B, W * n).gather(1, at)
    ended = (token == EOS) | st["done"].bool().gather(1, parent)
    return total.float(), parent.int(), token.int(), ended.to(torch.uint8)


def _run_reorder(st):
    c = st["case"]
    B, W, K, page, cols = c["B"], c["W"], c["K"], c["page"], st["cols"]
    if own:
        z = _library()
        if "layers" not in st:
            st["layers"] = z.make_pages_list(list(st["k"]), list(st["v"]))
        z.zsaa_op_beam_reorder(st["layers"], B, W, K, st["parent"], st["table"], st["table_out"], cols, st["lens"],
                               st["lens_out"], st["fresh"])
        return st["table_out"], st["lens_out"], st["k"], st["v"]
    slot = torch.arange(B * K, device="cuda")
    par = st["parent"].long()
    src = (par + W * torch.arange(B, device="cuda")[:, None]).reshape(-1)
    same = par[:, :, None] == par[:, None, :]
    again = torch.tril(same, diagonal=-1).any(2).reshape(-1)  # an earlier child has the parent's page
    lens = st["lens"][src].long()
    whole, part = lens // page, lens % page
    mine = st["table"][src].long()
    kept_page = mine.gather(1, whole[:, None])[:, 0]
    fresh = st["fresh"].long()
    new_page = torch.where(again | (part == 0), fresh, kept_page)
    col = torch.arange(cols, device="cuda")
    out = torch.where(col < whole[:, None], mine, torch.where(col == whole[:, None], new_page[:, None], -1))
    moved = (again & (part > 0))[:, None] & (torch.arange(page, device="cuda") < part[:, None])
    read = torch.where(again & (part > 0), kept_page, fresh)  # slots that copy nothing rewrite their own fresh page
    for pool in (st["k"], st["v"]):
        pool[:, fresh[slot]] = torch.where(moved[None, :, None, :, None], pool[:, read], pool[:, fresh[slot]])
    return out.int(), lens.int(), st["k"], st["v"]


# ------------------------------------------------------------------ from the definitions, in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return dict(append=_exact_append, attention=_exact_attention, select=_exact_select,
                reorder=_exact_reorder)[case["op"]](case, st)


def _exact_append(case, st):
    Hq, Hkv, hd, page = case["Hq"], case["Hkv"], case["hd"], case["page"]
    n, lens = _append_sizes(case)
    k, v, x = st["k"].double(), st["v"].double(), st["qkv"].double().reshape(st["T"], -1, hd)
    z = torch.complex(x[:, :Hq + Hkv, :hd // 2], x[:, :Hq + Hkv, hd // 2:])
    exponent = torch.arange(0, hd, 2, device="cuda", dtype=torch.float64) / hd
    turn = st["pos"].double()[:, None, None] * torch.exp(-exponent * math.log(case["theta"]))
    z = z * torch.polar(torch.ones_like(turn), turn)
    y = torch.cat([z.real, z.imag], dim=2)
    table = st["table"].tolist()
    t = 0
    for s in range(case["S"]):
        at = range(lens[s] - n[s], lens[s])
        pages = torch.tensor([table[s][i // page] for i in at], device="cuda")
        off = torch.tensor([i % page for i in at], device="cuda")
        k[pages, :, off] = y[t:t + n[s], Hq:]
        v[pages, :, off] = x[t:t + n[s], Hq + Hkv:]
        t += n[s]
    return y[:, :Hq], k, v


def _exact_attention(case, st):
    lens, plens, ends = _attention_sizes(case)
    S, nq, Hq, Hkv, hd, page = (case[x] for x in ("S", "nq", "Hq", "Hkv", "hd", "page"))
    out = torch.empty(S, nq, Hq, hd, dtype=torch.float64, device="cuda")
    lse = torch.empty(S, nq, Hq, dtype=torch.float64, device="cuda")

    def entries(pool, row, n):
        return pool[row[:-(-n // page)].long()].double().permute(1, 0, 2, 3).reshape(Hkv, -1, hd)[:, :n]

    group = -1
    for s in range(S):
        while case["G"] and (group < 0 or s >= ends[group + 1]):
            group += 1
            shared = [entries(p, st["ptable"][group], plens[group]) for p in (st["k"], st["v"])]
        kk, vv = (entries(p, st["table"][s], lens[s]) for p in (st["k"], st["v"]))
        if case["G"]:
            kk, vv = torch.cat([shared[0], kk], 1), torch.cat([shared[1], vv], 1)
        for j in range(nq):
            last = kk.shape[1] - nq + j + 1
            q = st["q"][s, j].double().reshape(Hkv, Hq // Hkv, hd)
            w = torch.einsum("gpd,gnd->gpn", q, kk[:, :last]) * hd ** -0.5
            out[s, j] = torch.einsum("gpn,gnd->gpd", torch.softmax(w, 2), vv[:, :last]).reshape(Hq, hd)
            lse[s, j] = torch.logsumexp(w, 2).reshape(Hq) * LOG2E
    return out, lse


def _exact_select(case, st):
    B, W, V, K = (case[x] for x in ("B", "W", "V", "K"))
    scores, parents, tokens, ended = [], [], [], []
    for b in range(B):
        found = []
        for w in range(W):
            if st["done"][b, w]:
                row = torch.full((V,), -math.inf, dtype=torch.float64, device="cuda")
                row[EOS] = 0.0
            else:
                row = st["logits"][b * W + w, :V].double()
                row = row - row.max()
                row = row - torch.log(torch.exp(row).sum())
            row = row + st["scores"][b, w].double()
            limit = torch.topk(row, min(K, V)).values[-1]
            for t in torch.nonzero(row >= limit)[:, 0].tolist() if limit > -math.inf else torch.topk(row, min(K, V)).indices.tolist():
                found.append((-float(row[t]), w, t))
        found.sort()
        scores.append([-f[0] for f in found[:K]])
        parents.append([f[1] for f in found[:K]])
        tokens.append([f[2] for f in found[:K]])
        ended.append([int(f[2] == EOS or st["done"][b, f[1]].item()) for f in found[:K]])
    return (torch.tensor(scores, dtype=torch.float64), torch.tensor(parents, dtype=torch.int32),
            torch.tensor(tokens, dtype=torch.int32), torch.tensor(ended, dtype=torch.uint8))


def _exact_reorder(case, st):
    B, W, K, page = (case[x] for x in ("B", "W", "K", "page"))
    k, v = st["k"].double(), st["v"].double()
    parent, table, lens, fresh = (st[x].tolist() for x in ("parent", "table", "lens", "fresh"))
    rows, out_lens = [], []
    for b in range(B):
        taken = set()
        for i, p in enumerate(parent[b]):
            s = b * W + p
            whole, part = divmod(lens[s], page)
            row = table[s][:whole]
            if part and p not in taken:
                row.append(table[s][whole])
            else:
                row.append(fresh[b * K + i])
                for pool in (k, v):
                    pool[:, row[-1], :, :part] = pool[:, table[s][whole], :, :part]
            taken.add(p)
            rows.append(row + [-1] * (st["cols"] - len(row)))
            out_lens.append(lens[s])
    return (torch.tensor(rows, dtype=torch.int32), torch.tensor(out_lens, dtype=torch.int32), k, v)
