"""Drafted tokens and the pages behind them, as measurable cases.

Four operators that a serving loop uses around its attention over paged caches:

* ``verify``   which drafted tokens stand against the target's probabilities, and the
               token that follows them, from given random numbers.
* ``resize``   page tables that grow and shrink over a count of references per page.
* ``fork``     new sequences that continue others from some length on: whole pages
               shared, the partly filled one copied.
* ``compact``  the chosen entries of a sequence moved together, in place or into
               other pages (a pruned cache, the accepted path of a draft tree).

Cache pages are ``[layer][page, KV head, entry, dim]``; a table row lists a sequence's
pages in order, -1 past its last one.  Layer sizes are those of the repository's 1B, 8B
and float32 configurations (``inputs.py``) or generic ones.  Lengths of a ragged batch
follow from the case alone, every value from the seed.

Where ``own`` is false, ``run`` computes the same in elementary torch operations;
probabilities and their running sums are in 64 bits, because the token that a random
number picks lies next to a border of such a sum.
"""

from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

CACHE_1B = dict(Hkv=8, hd=64, dtype="bf16")
CACHE_8B = dict(Hkv=8, hd=128, dtype="bf16")
CACHE_F32 = dict(Hkv=4, hd=32, dtype="f32")


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # One interactive request with four drafted tokens: the smallest call, latency.
        dict(name="verify_s1_n4", op="verify", S=1, n=4, V=128256, pad=0, temp="one", masked=False, ragged=False, lookup=False,
             dtype="f32"),
        # A serving batch, five drafts each, every request with its own temperature (some 0).
        dict(name="verify_s64_n5", op="verify", S=64, n=5, V=128256, pad=0, temp="mixed", masked=False, ragged=False,
             lookup=False, dtype="f32"),
        # An odd vocabulary in padded bf16 rows, banned tokens, drafts that ended early.
        dict(name="verify_s24_n3_bf16", op="verify", S=24, n=3, V=50257, pad=15, temp="mixed", masked=True, ragged=True,
             lookup=False, dtype="bf16"),
        # Drafts looked up in the prompt (no draft model, so no draft probabilities).
        dict(name="verify_lookup_s16_n15", op="verify", S=16, n=15, V=32003, pad=5, temp="one", masked=False, ragged=True,
             lookup=True, dtype="f32"),
        # A step of 64 sequences: a few cross into a new page.
        dict(name="resize_step_s64", op="resize", S=64, low=700, high=705, page=16, n_pages=8192, shared=4, swap=False),
        # Prompts of up to 4000 tokens come and go over a pool that fills the card.
        dict(name="resize_turnover_s512", op="resize", S=512, low=0, high=4000, page=16, n_pages=131072, shared=8, swap=True),
        # Four samples of one short prompt, all layers of the 1B shape.
        dict(name="fork_1b_n4", op="fork", L=16, S=1, N=4, len=141, page=16, ragged=False, cut=False, **CACHE_1B),
        # Eight samples of each of 16 prompts of the 8B shape, some from the middle.
        dict(name="fork_8b_n128", op="fork", L=32, S=16, N=128, len=1190, page=64, ragged=True, cut=True, **CACHE_8B),
        # The accepted path of a tree of 25 drafts, 8 sequences, all layers of the 1B shape.
        dict(name="compact_path_1b", op="compact", L=16, S=8, len=421, tail=25, kept=6, page=16, ragged=False, moved=False,
             **CACHE_1B),
        # A cache of the 8B shape pruned to half of its entries, in place.
        dict(name="compact_half_8b", op="compact", L=32, S=8, len=2011, tail=0, kept=1003, page=64, ragged=True, moved=False,
             **CACHE_8B),
        # A long document pruned to a quarter, one layer with entries of its own, into other pages.
        dict(name="compact_document_8b", op="compact", L=1, S=1, len=65000, tail=0, kept=16250, page=32, ragged=False,
             moved=True, **CACHE_8B),
        # The float32 cache, pruned in place.
        dict(name="compact_f32", op="compact", L=2, S=12, len=413, tail=0, kept=200, page=16, ragged=True, moved=False,
             **CACHE_F32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cache(rng):
    if rng.random() < 0.2:
        return dict(Hkv=rng.choice([1, 4, 8]), hd=rng.choice([32, 64, 128]), dtype="f32")
    return dict(Hkv=rng.choice([8, 8, 4, 2, 1, 5, 12]), hd=rng.choice([64, 128]), dtype="bf16")


def draw(rng: random.Random):
    while True:
        case = _drawn(rng)
        if work(case)["bytes"] <= (360e6 if case["op"] == "verify" else 2e9):  # within the largest listed ones
            return case


def _drawn(rng):
    op = rng.choice(["verify", "verify", "resize", "fork", "compact", "compact"])
    page = rng.choice([16, 32, 64, 128])
    if op == "verify":
        return dict(op=op, S=_log_int(rng, 1, 96), n=rng.choice([0, 1, 2, 3, 4, 5, 7, 15]), V=_log_int(rng, 900, 128256),
                    pad=rng.randint(0, 9), temp=rng.choice(["one", "mixed"]), masked=rng.random() < 0.4,
                    ragged=rng.random() < 0.5, lookup=rng.random() < 0.25, dtype=rng.choice(["f32", "f32", "bf16"]))
    if op == "resize":
        S, high = _log_int(rng, 1, 600), _log_int(rng, 20, 6000)
        shared = rng.randint(0, 5)
        need = S * (-(-high // page) + 1)
        return dict(op=op, S=S, low=rng.choice([0, rng.randint(0, high), high - rng.randint(0, 8)]), high=high, page=page,
                    n_pages=need + rng.choice([0, rng.randint(0, 3 * need)]) + 8, shared=shared, swap=rng.random() < 0.5)
    if op == "fork":
        S = _log_int(rng, 1, 40)
        return dict(op=op, L=_log_int(rng, 1, 32), S=S, N=_log_int(rng, 1, 200), len=_log_int(rng, 1, 3000), page=page,
                    ragged=rng.random() < 0.6, cut=rng.random() < 0.4, **_cache(rng))
    n = _log_int(rng, 8, 30000)
    tail = rng.choice([0, 0, min(n, rng.randint(2, 60))])
    return dict(op=op, L=_log_int(rng, 1, 32), S=max(1, min(_log_int(rng, 1, 48), 200000 // n)), len=n, tail=tail,
                kept=rng.randint(1, tail or n), page=page, ragged=rng.random() < 0.6, moved=rng.random() < 0.3, **_cache(rng))


# ------------------------------------------------------------------ sizes that follow from a case

def _spread(case, n, most, salt):
    """n lengths: all `most`, or for a ragged case between half of it and it."""
    if not case["ragged"]:
        return [most] * n
    r = random.Random(1000003 * n + 101 * most + salt)
    return [r.randint(max(1, most - most // 2), most) if most else 0 for _ in range(n)]


def _esz(case):
    return 2 if case["dtype"] == "bf16" else 4


def _resize_lens(case):
    """Two sets of lengths that a batch goes to and fro between."""
    r = random.Random(31 * case["S"] + case["high"])
    if not case["swap"]:  # all sequences grow by some tokens and go back
        a = [r.randint(max(0, case["low"] - 40), case["low"]) for _ in range(case["S"])]
        return a, [x + case["high"] - case["low"] for x in a]
    # some sequences end while others, waiting so far, start
    a, b = [], []
    for _ in range(case["S"]):
        x, y = r.randint(1, case["high"]), r.randint(0, case["high"])
        a.append(x if r.random() < 0.5 else 0)
        b.append(0 if a[-1] and r.random() < 0.7 else y)
    return a, b


def _fork_sizes(case):
    """Lengths of the parents; of each child its parent and the entries that it takes."""
    lens = _spread(case, case["S"], case["len"], 7)
    r = random.Random(17 * case["N"] + case["len"])
    parent = [i % case["S"] for i in range(case["N"])]
    if case["ragged"]:
        r.shuffle(parent)
    at = [r.randint(1, lens[p]) if case["cut"] and r.random() < 0.5 else lens[p] for p in parent]
    return lens, parent, at


def _compact_sizes(case):
    """Lengths, first entries that may move, and entries kept from there on."""
    lens = _spread(case, case["S"], case["len"], 8)
    start = [max(0, n - case["tail"]) if case["tail"] else 0 for n in lens]
    r = random.Random(13 * case["S"] + case["kept"])
    room = [n - a for n, a in zip(lens, start)]
    return lens, start, [min(x, max(1, r.randint(case["kept"] // 2, case["kept"]) if case["ragged"] else case["kept"]))
                         for x in room]


def _entry(case):
    return 2 * case["Hkv"] * case["hd"] * _esz(case) * case["L"]


def work(case):
    op = case["op"]
    if op == "verify":
        S, n, V = case["S"], case["n"], case["V"]
        rows = S * (n + 1) + (0 if case["lookup"] else S * n)
        return dict(bytes=rows * V * _esz(case) + 4 * S * (5 * n + 7), flops=4 * rows * V)
    page = case["page"]
    if op == "resize":
        a, b = _resize_lens(case)
        touched = sum(abs(-(-x // page) - -(-y // page)) for x, y in zip(a, b))
        return dict(bytes=4 * case["n_pages"] + 12 * touched + 12 * case["S"], flops=0)
    if op == "fork":
        lens, _, at = _fork_sizes(case)
        moved = sum(x % page for x in at) * _entry(case)
        return dict(bytes=2 * moved + sum(16 * (x // page + 1) for x in at) + 12 * case["N"], flops=0)
    _, _, kept = _compact_sizes(case)
    return dict(bytes=2 * sum(kept) * _entry(case) + 4 * sum(kept) + 8 * (sum(kept) // page + case["S"]) + 16 * case["S"], flops=0)


# ------------------------------------------------------------------ inputs

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _free(n_pages, seed):
    free = list(range(n_pages))
    random.Random(seed).shuffle(free)
    return free


def _pool(g, n_pages, case):
    size = (case["L"], n_pages, case["Hkv"], case["page"], case["hd"])
    return [torch.randn(size, generator=g, device="cuda", dtype=_type(case)) for _ in range(2)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return dict(verify=_prepare_verify, resize=_prepare_resize, fork=_prepare_fork,
                compact=_prepare_compact)[case["op"]](case, seed, g)


def _prepare_verify(case, seed, g):
    S, n, V, ld = case["S"], case["n"], case["V"], case["V"] + case["pad"]
    rand = lambda *size: torch.rand(*size, generator=g, device="cuda")  # noqa: E731
    target = 3.0 * torch.randn(S, n + 1, ld, generator=g, device="cuda")
    # a smaller model's logits are near the target's: about two of three drafts stand
    draft = target[:, :n] + 0.8 * torch.randn(S, n, ld, generator=g, device="cuda")
    if case["masked"]:  # tokens that a grammar bans, in both
        banned = rand(S, 1, ld) < 0.3
        target.masked_fill_(banned, -math.inf)
        draft.masked_fill_(banned, -math.inf)
    target, draft = target.to(_type(case)), draft.to(_type(case))
    temp = None
    if case["temp"] == "mixed":
        temp = torch.tensor([0.0, 0.6, 0.8, 1.0, 1.3], device="cuda")[torch.randint(0, 5, (S,), generator=g, device="cuda")]
    t = torch.ones(S, device="cuda") if temp is None else temp
    rows = target[:, :n, :V] if case["lookup"] else draft[:, :, :V]
    noise = -torch.log(-torch.log(rand(S, n, V).clamp_(1e-9, 1 - 1e-7)))
    drafts = torch.argmax(rows.float() + t[:, None, None] * noise, dim=2).to(torch.int32) if n else torch.zeros(
        S, 0, dtype=torch.int32, device="cuda")
    if case["lookup"]:  # what followed last time is often, not always, what follows now
        drafts = torch.where(rand(S, n) < 0.8, drafts, torch.randint(0, V, (S, n), generator=g, device="cuda").to(torch.int32))
    if case["ragged"] and n:  # -1: the draft model stopped before
        drafts = torch.where(torch.arange(n, device="cuda") < torch.randint(0, n + 1, (S, 1), generator=g, device="cuda"), drafts, -1)
    lens = torch.randint(n + 1, 3000, (S,), generator=g, device="cuda").to(torch.int32)
    new = lambda *size, dtype=torch.int32: torch.empty(*size, dtype=dtype, device="cuda")  # noqa: E731
    return dict(case=case, target=target, draft=None if case["lookup"] else draft, drafts=drafts.to(torch.int32).contiguous(),
                temp=temp, uniform=rand(S, n + 1), lens=lens, accepted=new(S), tokens=new(S, n + 1),
                logp=new(S, n + 1, dtype=torch.float32), lens_out=new(S))


def _prepare_resize(case, seed, g):
    S, page, n_pages, shared = case["S"], case["page"], case["n_pages"], case["shared"]
    a, b = _resize_lens(case)
    cols = max(-(-x // page) for x in a + b) + 1
    free, refs = _free(n_pages, seed), np.zeros(n_pages, np.int32)
    table = np.full((S, cols), -1, np.int32)
    for s, n in enumerate(a):
        used = -(-n // page)
        first = s - s % 4  # four sequences in a row have a prompt in common
        same = min(shared, used, -(-a[first] // page) if first < s else 0)
        table[s, :same] = table[first, :same]
        table[s, same:used] = [free.pop() for _ in range(used - same)]
        np.add.at(refs, table[s, :used], 1)
    return dict(case=case, refs=_ints(refs), table=_ints(table), cols=cols, lens=_ints(a), goals=[_ints(b), _ints(a)],
                lens_out=_ints(a), n_free=_ints([0]))


def _prepare_fork(case, seed, g):
    page, N = case["page"], case["N"]
    lens, parent, at = _fork_sizes(case)
    cols = max(-(-x // page) for x in lens) + 2
    n_pages = sum(-(-x // page) for x in lens) + N + 3
    free, refs = _free(n_pages, seed), np.zeros(n_pages, np.int32)
    table = np.full((case["S"], cols), -1, np.int32)
    for s, n in enumerate(lens):
        used = -(-n // page)
        table[s, :used] = [free.pop() for _ in range(used)]
        refs[table[s, :used]] = 1
    k, v = _pool(g, n_pages, case)
    return dict(case=case, k=k, v=v, refs=_ints(refs), n_pages=n_pages, table=_ints(table), cols=cols, lens=_ints(lens),
                parent=_ints(parent), at=_ints(at) if case["cut"] else None, none=_ints([0] * N),
                table_out=torch.full((N, cols), -1, dtype=torch.int32, device="cuda"), lens_out=_ints([0] * N),
                spare=_ints([0] * N), n_free=_ints([0]))


def _prepare_compact(case, seed, g):
    page, S = case["page"], case["S"]
    lens, start, kept = _compact_sizes(case)
    r = np.random.RandomState(seed % (1 << 32))
    width = max(kept) + 1
    keep = np.full((S, width), -1, np.int32)
    for s in range(S):
        keep[s, :kept[s]] = start[s] + np.sort(r.permutation(lens[s] - start[s])[:kept[s]])
    cols = max(-(-x // page) for x in lens) + 1
    ends = [a + b for a, b in zip(start, kept)]
    out_cols = max(-(-x // page) for x in ends) + 1 if case["moved"] else cols
    n_pages = sum(-(-x // page) for x in lens) + (sum(-(-x // page) for x in ends) if case["moved"] else 0) + 2
    free = _free(n_pages, seed)
    rows = lambda lens, cols: _ints([[free.pop() for _ in range(-(-x // page))] + [-1] * (cols - -(-x // page)) for x in lens])  # noqa: E731
    table = rows(lens, cols)
    k, v = _pool(g, n_pages, case)
    return dict(case=case, k=k, v=v, table=table, cols=cols, lens=_ints(lens), start=_ints(start) if case["tail"] else None,
                first=_ints(start), keep=_ints(keep), width=width, n_keep=_ints(kept), out_cols=out_cols,
                table_out=rows(ends, out_cols) if case["moved"] else table, lens_out=_ints([0] * S), total=sum(kept))


# ------------------------------------------------------------------ one pass

def run(state):
    return dict(verify=_run_verify, resize=_run_resize, fork=_run_fork, compact=_run_compact)[state["case"]["op"]](state)


def _library():
    from paper_2509_01190_gb300 import zsaa
    return zsaa


def _log_softmax(x, t, greedy):
    """Of rows x [S, rows, V] in 64 bits at temperature t [S]; greedy [S]: all on the first maximum."""
    top = x.amax(2, keepdim=True)
    place = torch.arange(x.shape[2], device="cuda")
    first = torch.where(x == top, place, x.shape[2]).amin(2, keepdim=True)
    y = (x - top) / t[:, None, None]
    y = y - torch.log(torch.exp(y).sum(2, keepdim=True))
    return torch.where(greedy[:, None, None], torch.where(place == first, 0.0, -math.inf), y)


def _run_verify(st):
    c = st["case"]
    S, n, V = c["S"], c["n"], c["V"]
    if own:
        z = _library()
        if "ws" not in st:
            st["ws"] = torch.empty(z.zsaa_op_draft_verify_workspace(S, n, V), dtype=torch.uint8, device="cuda")
        ld = V + c["pad"]
        z.zsaa_op_draft_verify(st["target"], ld, st["draft"], ld, z.ZSAA_F32 if c["dtype"] == "f32" else z.ZSAA_BF16, S, n, V,
                               st["drafts"], st["temp"], st["uniform"], st["accepted"], st["tokens"], st["logp"], st["lens"],
                               st["lens_out"], st["ws"], st["ws"].numel())
        return st["accepted"], st["tokens"], st["logp"], st["lens_out"]
    seq = torch.arange(S, device="cuda")
    u = st["uniform"].double()
    t = torch.ones(S, device="cuda", dtype=torch.float64) if st["temp"] is None else st["temp"].double()
    greedy = t == 0
    t = torch.where(greedy, 1.0, t)
    lp = _log_softmax(st["target"][:, :, :V].double(), t, greedy)
    x = st["drafts"].long()
    there = torch.cumprod((x >= 0).long(), 1).bool()
    x = x.clamp(min=0)
    at = x[:, :, None]
    px = torch.exp(lp[:, :n].gather(2, at)[..., 0])
    if st["draft"] is None:
        qx = torch.ones_like(px)
    else:
        lq = _log_softmax(st["draft"][:, :, :V].double(), t, greedy)
        qx = torch.exp(lq.gather(2, at)[..., 0])
    stands = there & (u[:, :n] * qx < px)
    a = torch.cumprod(stands.long(), 1).sum(1)
    p = torch.exp(lp[seq, a])
    if n:
        j = a.clamp(max=n - 1)
        if st["draft"] is None:
            q = torch.where(torch.arange(V, device="cuda") == x[seq, j][:, None], 1.0, 0.0)
        else:
            q = torch.exp(lq[seq, j])
        refused = (a < n) & there[seq, j]
        r = torch.where(refused[:, None], torch.clamp(p - q, min=0.0), p)
        r = torch.where(r.sum(1, keepdim=True) > 0, r, p)
    else:
        r = p
    c_sum = torch.cumsum(r, 1)
    token = (c_sum <= u[:, n:] * c_sum[:, -1:]).sum(1)
    col = torch.arange(n + 1, device="cuda")
    both = torch.cat([x, token[:, None]], 1)
    both = torch.where(col == a[:, None], token[:, None], both)
    logp = lp.gather(2, both[:, :, None])[..., 0]
    tokens = torch.where(col <= a[:, None], both, -1).int()
    return a.int(), tokens, torch.where(col <= a[:, None], logp, 0.0).float(), (st["lens"] - n + a).int()


def _resized(refs, page, table, lens, want):
    """Plain resize: refs and table in place; the lengths reached and the free pages left."""
    n_pages, cols = refs.shape[0], table.shape[1]
    col = torch.arange(cols, device="cuda")
    old, new = (-(-x // page) for x in (lens.long(), want.long()))
    gone = (col >= new[:, None]) & (col < old[:, None])
    refs.index_add_(0, torch.where(gone, table, 0).reshape(-1).long(), -gone.reshape(-1).int())
    need = (col >= old[:, None]) & (col < new[:, None])
    got, n_free = _taken(refs, table, need)
    return torch.where(new > old, torch.minimum(want.long(), (old + got) * page), want.long()).int(), n_free


def _taken(refs, table, need):
    """The free pages, lowest first, to the table's places that need one, row by row."""
    free = refs == 0
    n_free = free.sum()
    listed = torch.zeros_like(refs, dtype=torch.int64)
    listed.scatter_add_(0, torch.where(free, torch.cumsum(free.int(), 0) - 1, 0),
                        torch.where(free, torch.arange(refs.shape[0], device="cuda"), 0))
    rank = (torch.cumsum(need.reshape(-1).int(), 0) - 1).reshape(need.shape)
    given = need & (rank < n_free)
    page = listed[rank.clamp(0, refs.shape[0] - 1)]
    table.copy_(torch.where(given, page.int(), table))
    refs.index_add_(0, torch.where(given, page, 0).reshape(-1), given.reshape(-1).int())
    return given.sum(1), (n_free - given.sum()).int().reshape(1)


def _run_resize(st):
    c = st["case"]
    st["goals"].reverse()  # a batch that goes to and fro between two sets of lengths
    want = st["goals"][1]
    st["lens"], st["lens_out"] = st["lens_out"], st["lens"]
    if own:
        z = _library()
        z.zsaa_op_paged_resize(st["refs"], c["n_pages"], c["page"], c["S"], st["table"], st["cols"], st["lens"], want,
                               st["lens_out"], st["n_free"])
        return st["table"], st["refs"], st["lens_out"], st["n_free"]
    lens_out, n_free = _resized(st["refs"], c["page"], st["table"], st["lens"], want)
    st["lens_out"].copy_(lens_out)
    return st["table"], st["refs"], st["lens_out"], n_free


def _run_fork(st):
    """The last samples give their pages back, the next ones continue the parents."""
    c = st["case"]
    page, N, cols = c["page"], c["N"], st["cols"]
    if own:
        z = _library()
        if "layers" not in st:
            st["layers"] = z.make_pages_list(list(st["k"]), list(st["v"]))
        z.zsaa_op_paged_resize(st["refs"], st["n_pages"], page, N, st["table_out"], cols, st["lens_out"], st["none"], st["spare"])
        z.zsaa_op_paged_fork(st["layers"], st["refs"], c["S"], st["table"], cols, st["lens"], N, st["parent"], st["at"],
                             st["table_out"], st["lens_out"], st["n_free"])
        return st["table_out"], st["lens_out"], st["n_free"], st["refs"], st["k"], st["v"]
    _resized(st["refs"], page, st["table_out"], st["lens_out"], st["none"])
    par = st["parent"].long()
    lens = st["lens"][par].long()
    if st["at"] is not None:
        lens = torch.minimum(lens, st["at"].long())
    whole, part = lens // page, lens % page
    mine = st["table"][par]
    col = torch.arange(cols, device="cuda")
    shared = col < whole[:, None]
    st["refs"].index_add_(0, torch.where(shared, mine, 0).reshape(-1).long(), shared.reshape(-1).int())
    st["table_out"].copy_(torch.where(shared, mine, st["table_out"]))
    got, n_free = _taken(st["refs"], st["table_out"], (col == whole[:, None]) & (part > 0)[:, None])
    part = torch.where(got > 0, part, 0)
    st["lens_out"].copy_(whole * page + part)
    some = part > 0
    src, dst = (torch.masked_select(t.gather(1, whole[:, None])[:, 0], some).long() for t in (mine, st["table_out"]))
    moved = (torch.arange(page, device="cuda") < torch.masked_select(part, some)[:, None])[None, :, None, :, None]
    for pool in (st["k"], st["v"]):
        pool[:, dst] = torch.where(moved, pool[:, src], pool[:, dst])
    return st["table_out"], st["lens_out"], n_free, st["refs"], st["k"], st["v"]


def _run_compact(st):
    c = st["case"]
    page, S = c["page"], c["S"]
    if own:
        z = _library()
        if "layers" not in st:
            st["layers"] = z.make_pages_list(list(st["k"]), list(st["v"]))
        z.zsaa_op_paged_compact(st["layers"], None, S, st["table"], st["cols"], st["lens"], st["start"], st["keep"], st["width"],
                                st["n_keep"], st["table_out"], st["out_cols"], st["lens_out"])
        return st["lens_out"], st["k"], st["v"]
    j = torch.arange(st["width"], device="cuda")
    live = (j < st["n_keep"][:, None]).reshape(-1)
    seq = torch.masked_select(torch.arange(S, device="cuda").repeat_interleave(st["width"], output_size=S * st["width"]), live)
    src = torch.masked_select(st["keep"].reshape(-1), live).long()
    dst = torch.masked_select((st["first"][:, None] + j).reshape(-1), live).long()
    from_page, to_page = st["table"][seq, src // page].long(), st["table_out"][seq, dst // page].long()
    for pool in (st["k"], st["v"]):
        pool[:, to_page, :, dst % page] = pool[:, from_page, :, src % page]
    return (st["first"] + st["n_keep"]).int(), st["k"], st["v"]


# ------------------------------------------------------------------ from the definitions, in 64 bits

def exact(case, seed):
    if case["op"] == "resize":
        return None  # page numbers alone
    st = prepare(case, seed)
    return dict(verify=_exact_verify, fork=_exact_fork, compact=_exact_compact)[case["op"]](case, st)


def _exact_verify(case, st):
    S, n, V = case["S"], case["n"], case["V"]
    accepted, tokens, logps = [], [], []
    for s in range(S):
        t = 1.0 if st["temp"] is None else float(st["temp"][s])
        u, x = st["uniform"][s].tolist(), st["drafts"][s].tolist()

        def probabilities(row):
            row = row[:V].double()
            if t == 0:
                p = torch.zeros_like(row)
                p[int(torch.nonzero(row == row.max())[0])] = 1.0
                return p
            return torch.softmax(row / t, 0)

        out, lp, left = [], [], None
        for j in range(n + 1):
            p = probabilities(st["target"][s, j])
            if j == n or x[j] < 0:
                left = p
                break
            if st["draft"] is None:
                q = torch.zeros_like(p)
                q[x[j]] = 1.0
            else:
                q = probabilities(st["draft"][s, j])
            if u[j] * float(q[x[j]]) < float(p[x[j]]):
                out.append(x[j])
                lp.append(math.log(float(p[x[j]])))
                continue
            left = torch.clamp(p - q, min=0)
            left = left if float(left.sum()) > 0 else p
            break
        accepted.append(len(out))
        sums = torch.cumsum(left, 0)
        out.append(int(torch.nonzero(sums > u[n] * sums[-1])[0]))
        lp.append(math.log(float(p[out[-1]])))
        tokens.append(out + [-1] * (n + 1 - len(out)))
        logps.append(lp + [0.0] * (n + 1 - len(lp)))
    a = torch.tensor(accepted, dtype=torch.int32)
    return a, torch.tensor(tokens, dtype=torch.int32), torch.tensor(logps, dtype=torch.float64), st["lens"].cpu() - n + a


def _exact_fork(case, st):
    page = case["page"]
    lens, parent, at = _fork_sizes(case)
    k, v = st["k"].double(), st["v"].double()
    table, refs = st["table"].tolist(), st["refs"].tolist()
    for p, m in zip(parent, at):
        for page_no in table[p][:m // page]:
            refs[page_no] += 1
    free = [i for i, c in enumerate(refs) if c == 0][::-1]
    rows = []
    for p, m in zip(parent, at):
        row = table[p][:m // page]
        if m % page:
            row.append(free.pop())
            refs[row[-1]] = 1
            for pool in (k, v):
                pool[:, row[-1], :, :m % page] = pool[:, table[p][m // page], :, :m % page]
        rows.append(row + [-1] * (st["cols"] - len(row)))
    whole = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return whole(rows), whole(at), whole([len(free)]), whole(refs), k, v


def _exact_compact(case, st):
    page = case["page"]
    _, start, kept = _compact_sizes(case)
    k, v = st["k"].double(), st["v"].double()
    for s in range(case["S"]):
        src = st["keep"][s, :kept[s]].long()
        dst = torch.arange(start[s], start[s] + kept[s], device="cuda")
        a, b = st["table"][s][src // page].long(), st["table_out"][s][dst // page].long()
        for pool in (k, v):
            pool[:, b, :, dst % page] = pool[:, a, :, src % page].clone()
    return torch.tensor([a + b for a, b in zip(start, kept)], dtype=torch.int32), k, v
