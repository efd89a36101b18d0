"""Paged caches on the GPU: appending with rotation and attention over shared prefixes,
against plain 64-bit forms.  Every pool starts as NaN, so an entry read that no query
sees, or one written that no row owns, shows."""

import random

import numpy as np
import pytest
import torch

import paged_ref as R
from helpers import need_gpu, np64

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _gpu(zlib):
    need_gpu()
    yield
    zlib.zsaa_device_status()


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Pool:
    """A NaN pool that gives out pages in a scattered order."""

    def __init__(self, z, dtype, Hkv, hd, page, n_pages, seed=0):
        self.z, self.page = z, page
        self.k, self.v = (torch.full((n_pages, Hkv, page, hd), float("nan"), device="cuda", dtype=DTYPES[dtype])
                          for _ in range(2))
        self.pages = z.make_pages(self.k, self.v)
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.free = list(range(n_pages))
        random.Random(seed).shuffle(self.free)

    def row(self, n, cols, fill=True):
        """A table row of n entries, their keys and values drawn (fill) or left NaN."""
        used = [self.free.pop() for _ in range(-(-n // self.page))]
        if fill and used:
            for pool in (self.k, self.v):
                at = torch.tensor(used, device="cuda")
                x = torch.randn((len(used),) + pool.shape[1:], generator=self.g, device="cuda").to(pool.dtype)
                if n % self.page:
                    x[-1, :, n % self.page:] = float("nan")
                pool[at] = x
        return used + [-1] * (cols - len(used))

    def np(self):
        return np64(self.k), np64(self.v)


def attend(z, p, q, table, lens, groups=None, ptable=None, plens=None, stream=None, ws=None, out=None, lse=None):
    S, n_q, Hq, _ = q.shape
    G = 0 if groups is None else len(groups) - 1
    cols, pcols = len(table[0]), len(ptable[0]) if G else 0
    n = z.zsaa_op_paged_attention_workspace(p.pages, S, n_q, Hq, G, cols, pcols)
    if ws is None:  # NaN bytes: what a call reads of its workspace it has written before
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full((S, n_q, Hq), 7.0, device="cuda") if lse is None else lse
    z.zsaa_op_paged_attention(p.pages, q, S, n_q, Hq, ints(table), cols, ints(lens), ints(groups) if G else None, G,
                              ints(ptable) if G else None, pcols, ints(plens) if G else None, out, lse, ws, ws.numel(),
                              stream=stream)
    return out, lse


def build(z, dtype, Hq, Hkv, hd, page, lens, n_q, groups=None, plens=(), seed=0, spare=1):
    cols = max(1, max(-(-n // page) for n in lens)) + spare
    pcols = max([1] + [-(-n // page) for n in plens])
    n_pages = sum(-(-n // page) for n in [*lens, *plens]) + 2
    p = Pool(z, dtype, Hkv, hd, page, n_pages, seed)
    table = [p.row(n, cols) for n in lens]
    ptable = [p.row(n, pcols) for n in plens]
    q = (1.5 * torch.randn(len(lens), n_q, Hq, hd, generator=p.g, device="cuda")).to(DTYPES[dtype])
    return p, q, table, ptable or None


def check(p, q, table, lens, out, lse, groups=None, ptable=None, plens=None):
    k, v = p.np()
    w = {}
    ref, ref_lse = R.attention(k, v, np64(q), table, lens, groups, ptable, plens, weighted=w)
    keys = max(lens) + (max(plens) if plens else 0) + 1
    tol, tol_lse = R.attention_tol(ref, w, keys, q.shape[-1], q.dtype == torch.bfloat16)
    got, got_lse = np64(out), np64(lse)
    pad = np.isnan(ref_lse)
    assert np.all(got[pad] == 7.0) and np.all(got_lse[pad] == 7.0), "padding rows were written"
    live = ~pad
    err = np.abs(got[live] - ref[live])
    assert np.all(err <= tol[live]), (float(np.nanmax(err / tol[live])), float(np.nanmax(err)))
    none = np.isneginf(ref_lse)
    assert np.all(np.isneginf(got_lse[none])) and np.all(got[none] == 0.0)
    some = live & ~none
    err = np.abs(got_lse[some] - ref_lse[some])
    assert np.all(err <= tol_lse + 2.0 ** -22 * np.abs(ref_lse[some])), float(err.max())


CASES = [
    # dtype, Hq, Hkv, hd, page, n_q, lens, groups, plens
    ("bf16", 8, 2, 64, 16, 1, [1], None, None),
    ("bf16", 4, 4, 128, 16, 1, [1, 0, 17, 33], None, None),
    ("bf16", 8, 1, 128, 32, 1, [127, 128, 129, 16, 15], None, None),
    ("bf16", 32, 8, 64, 16, 1, [21, 5, 9, 21], [0, 4], [99]),
    ("bf16", 32, 8, 128, 64, 1, [70, 1, 0, 140], [0, 3, 4], [0, 257]),
    ("bf16", 6, 2, 128, 256, 1, [300, 2], [0, 1, 2], [511, 1]),
    ("bf16", 10, 2, 64, 16, 3, [40, 3, 2, 1, 0], [0, 2, 2, 5], [64, 31, 130]),
    ("bf16", 7, 1, 64, 32, 16, [16, 200, 7], [0, 3], [300]),
    ("bf16", 8, 2, 128, 16, 2, [2, 90, 3, 4], [1, 3], [48]),            # first and last sequence are padding
    ("bf16", 4, 1, 64, 16, 1, [9] * 70, [0, 40, 70], [200, 333]),       # many rows to a prefix
    ("bf16", 12, 3, 128, 16, 1, [5] * 45, [0, 45], [1100]),
    ("bf16", 32, 8, 128, 128, 1, [6000], None, None),                   # one sequence over all SMs
    ("bf16", 8, 2, 64, 16, 5, [33] * 9, [0, 9], [4100]),
    ("bf16", 16, 16, 64, 16, 1, [100, 1, 63, 64, 65, 31], [0, 0, 6], [40, 16]),
    ("bf16", 16, 2, 64, 16, 16, [16, 100, 3, 0], None, None),            # 128 rows of one sequence
    ("bf16", 8, 1, 128, 32, 9, [9, 257, 30], [0, 2, 3], [128, 129]),
    ("bf16", 5, 1, 64, 64, 3, [70, 3, 2], None, None),
    ("bf16", 8, 1, 64, 16, 3, [5, 40], [0, 2], [12000]),                 # more than 32 partial results to a row
    ("bf16", 20, 1, 128, 16, 1, [3] * 70, list(range(71)), [17] * 70),  # more than 32 groups
    ("bf16", 10, 5, 64, 16, 1, [33, 0, 1, 90, 16] * 14, None, None),     # more CTAs than the SMs hold
    ("bf16", 10, 5, 128, 16, 3, [40, 1, 0, 17, 66] * 14, [0, 30, 70], [50, 0]),
    ("f32", 10, 5, 32, 16, 1, [33, 0, 1, 90, 16] * 14, None, None),
    ("f32", 10, 5, 64, 16, 2, [40, 1, 0, 17, 66] * 14, [2, 70], [35]),
    ("f32", 10, 5, 128, 16, 1, [33, 0, 1, 90, 16] * 14, [0, 40, 70], [0, 21]),
    ("f32", 4, 4, 32, 16, 1, [1, 0, 50], None, None),
    ("f32", 2, 1, 64, 16, 1, [3] * 40, list(range(41)), [17] * 40),
    ("f32", 4, 4, 32, 16, 3, [77, 3, 12, 40], [0, 1, 4], [413, 100]),
    ("f32", 8, 2, 64, 32, 1, [33, 64, 31], [0, 2, 3], [200, 0]),
    ("f32", 9, 3, 128, 16, 2, [2, 1, 130], [0, 3], [65]),
    ("f32", 4, 1, 128, 64, 1, [2500], None, None),
    ("f32", 16, 2, 64, 16, 4, [30] * 12, [0, 11, 12], [700, 20]),
]


def widened(rows, cols):
    """Table rows with room for more: what the call is planned for is the tables' width."""
    return None if rows is None else [r + [-1] * (cols - len(r)) for r in rows]


def rooms(dtype, page, groups):
    """Widths of the two tables, in pages.  A call over narrow tables takes one launch, one
    over wide ones is split over the SMs; entries with more than 16 rows to a KV head then
    take 128-row tiles, by the prefixes' tables alone or (rows of one sequence) by both."""
    some, many = 2100 // page, 64000 // page
    wide = [(some, some)] + ([(many, many)] if dtype == "bf16" else [])
    return [(0, 0)] + wide + ([(0, w) for _, w in wide] if groups is not None else [])


ROOMY = [c + (r,) for c in CASES for r in rooms(c[0], c[4], c[7])]


@pytest.mark.parametrize("dtype,Hq,Hkv,hd,page,n_q,lens,groups,plens,room", ROOMY)
def test_attention(zlib, dtype, Hq, Hkv, hd, page, n_q, lens, groups, plens, room):
    p, q, table, ptable = build(zlib, dtype, Hq, Hkv, hd, page, lens, n_q, groups, plens or ())
    table, ptable = widened(table, room[0]), widened(ptable, room[1])
    out, lse = attend(zlib, p, q, table, lens, groups, ptable, plens)
    check(p, q, table, lens, out, lse, groups, ptable, plens)
    again, lse2 = attend(zlib, p, q, table, lens, groups, ptable, plens)
    assert torch.equal(out, again) and torch.equal(lse, lse2), "two runs differ"


@pytest.mark.parametrize("seed", range(16))
def test_attention_of_drawn_sizes(zlib, seed):
    r = random.Random(seed)
    dtype = r.choice(["bf16", "bf16", "f32"])
    hd = r.choice([64, 128] if dtype == "bf16" else [32, 64, 128])
    Hkv, per, n_q, S = r.randint(1, 5), r.randint(1, 8), r.randint(1, 6), r.randint(1, 20)
    lens = [r.randint(0, 150) for _ in range(S)]
    G = r.randint(1, 4)
    groups = sorted(r.randint(0, S) for _ in range(G + 1))
    plens = [r.choice([0, r.randint(1, 900)]) for _ in range(G)]
    p, q, table, ptable = build(zlib, dtype, Hkv * per, Hkv, hd, r.choice([16, 64]), lens, n_q, groups, plens, seed)
    if seed % 3 == 1:
        ptable = widened(ptable, 5000)
    elif seed % 3 == 2:
        table, ptable = widened(table, 200), widened(ptable, 200)
    out, lse = attend(zlib, p, q, table, lens, groups, ptable, plens)
    check(p, q, table, lens, out, lse, groups, ptable, plens)


@pytest.mark.parametrize("dtype,cols", [("bf16", 10), ("bf16", 100), ("bf16", 5000), ("f32", 4), ("f32", 100)])
def test_a_later_draft_that_is_not_finite_stays_out_of_earlier_ones(zlib, dtype, cols):
    lens, n_q = [20, 4, 35], 4
    p, q, table, ptable = build(zlib, dtype, 20, 2, 64, 16, lens, n_q, [0, 3], [50])
    table, ptable = widened(table, cols), widened(ptable, cols)
    for s, n in enumerate(lens):  # the newest entry of every sequence
        page, off = table[s][(n - 1) // 16], (n - 1) % 16
        p.k[page, :, off] = float("nan")
        p.v[page, :, off] = float("inf")
    out, lse = attend(zlib, p, q, table, lens, [0, 3], ptable, [50])
    assert torch.isfinite(out[:, :-1]).all() and not torch.isfinite(out[:, -1]).any()
    clean = [n - 1 for n in lens]  # the first three queries alone
    check(p, q[:, :-1].contiguous(), table, clean, out[:, :-1].contiguous(), lse[:, :-1].contiguous(), [0, 3], ptable, [50])


NAN_BITS = {"f32": (0x7fffffff, -1, 0x7fc00000, 0x7f800001), "bf16": (0x7fff, -1, 0x7fc0, 0x7f81)}


@pytest.mark.parametrize("dtype,hd,cols", [("f32", 32, 0), ("f32", 32, 300), ("f32", 64, 0), ("f32", 64, 300), ("f32", 128, 0),
                                           ("f32", 128, 300), ("bf16", 64, 0), ("bf16", 128, 300), ("bf16", 64, 5000),
                                           ("bf16", 128, 5000)])
@pytest.mark.parametrize("place", ["query", "own key", "own value", "prefix key", "prefix value"])
def test_a_nan_that_a_query_sees_reaches_its_result(zlib, dtype, hd, cols, place):
    """Any NaN, CUDA's own 0x7fffffff among them; rows that do not see it keep their bits."""
    lens, plens, groups = [23, 9, 30], [40, 18], [0, 2, 3]
    p, q, table, ptable = build(zlib, dtype, 12, 2, hd, 16, lens, 3, groups, plens)
    table, ptable = widened(table, cols), widened(ptable, cols)
    clean, clean_lse = attend(zlib, p, q, table, lens, groups, ptable, plens)
    bits = torch.int32 if dtype == "f32" else torch.int16
    for nan in NAN_BITS[dtype]:
        rows = (ptable[0] if place.startswith("prefix") else table[2])[0]
        if place == "query":
            word = q.view(bits)[1, 2, 7:8, hd - 3]
        else:
            word = (p.k if place.endswith("key") else p.v).view(bits)[rows, 1, 5:6, 11]
        before = word.clone()
        word.fill_(nan)
        out, lse = attend(zlib, p, q, table, lens, groups, ptable, plens)
        k, v = p.np()
        ref, ref_lse = R.attention(k, v, np64(q), table, lens, groups, ptable, plens)
        hit, hit_lse = torch.from_numpy(np.isnan(ref)).cuda(), torch.from_numpy(np.isnan(ref_lse)).cuda()
        assert hit.any() and not hit.all()
        assert torch.equal(torch.isnan(out), hit) and torch.equal(torch.isnan(lse), hit_lse), hex(nan)
        assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit_lse], clean_lse[~hit_lse])
        word.copy_(before)


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_large_scores(zlib, dtype, hd):
    """Scores far apart, rising and falling along the keys: the running maximum moves
    from block to block."""
    for sign, n_q, cols in ((1.0, 1, 50), (-1.0, 1, 50), (1.0, 1, 500), (-1.0, 1, 500), (1.0, 5, 20000), (-1.0, 5, 20000)):
        p, q, table, _ = build(zlib, dtype, 4, 1, hd, 16, [700], n_q, seed=3)
        table = widened(table, cols)
        ramp = torch.linspace(0.0, 40.0, 700, device="cuda")
        for i in range(700):
            p.k[table[0][i // 16], :, i % 16] = sign * ramp[i] * (hd ** -0.5) * torch.sign(q[0, 0, 0]).to(p.k.dtype)
        out, lse = attend(zlib, p, q, table, [700])
        check(p, q, table, [700], out, lse)


@pytest.mark.parametrize("dtype,cols", [("bf16", 0), ("bf16", 100), ("bf16", 5000), ("f32", 0), ("f32", 100)])
def test_attention_without_lse_on_another_stream_and_as_two_graphs(zlib, dtype, cols):
    lens, groups, plens = [40, 3, 66], [0, 2, 3], [90, 300]
    p, q, table, ptable = build(zlib, dtype, 40, 2, 128, 16, lens, 1, groups, plens)
    ptable = widened(ptable, cols)
    want, want_lse = attend(zlib, p, q, table, lens, groups, ptable, plens)
    t, l, g, pt, pl = ints(table), ints(lens), ints(groups), ints(ptable), ints(plens)
    n = zlib.zsaa_op_paged_attention_workspace(p.pages, 3, 1, 40, 2, len(table[0]), len(ptable[0]))

    def call(out, lse, ws):
        zlib.zsaa_op_paged_attention(p.pages, q, 3, 1, 40, t, len(table[0]), l, g, 2, pt, len(ptable[0]), pl, out, lse, ws,
                                     ws.numel())

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out, ws = torch.empty_like(q), torch.empty(n, dtype=torch.uint8, device="cuda")
        call(out, None, ws)
    side.synchronize()
    assert torch.equal(out, want)
    runs = []
    for _ in range(2):
        out, lse, ws = torch.empty_like(q), torch.empty_like(want_lse), torch.empty(n, dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out, lse, ws)
        runs.append((graph, out, lse, ws))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (graph, out, lse, ws), s in zip(runs, streams):
            with torch.cuda.stream(s):
                out.zero_()
                lse.zero_()
                ws.fill_(255)
                graph.replay()
    torch.cuda.synchronize()
    for _, out, lse, _ in runs:
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    # a replay reads the lengths that are there then
    l.copy_(ints([12, 1, 50]))
    runs[0][0].replay()
    torch.cuda.synchronize()
    # (entries past the new lengths are not NaN here, the reference does not read them)
    check(p, q, table, [12, 1, 50], runs[0][1], runs[0][2], groups, ptable, plens)


@pytest.mark.parametrize("hd", [64, 128])
def test_128_row_tiles_between_other_tensor_core_kernels(zlib, hd):
    """Projections and attention launched one behind the other, as a layer has them: each
    kernel may start before the one ahead has ended, and all of them take tensor memory."""
    lens, plens, groups, Hq, Hkv, d = [20] * 24, [2100, 1500], [0, 9, 24], 16, 2, 256
    p, q, table, ptable = build(zlib, "bf16", Hq, Hkv, hd, 16, lens, 1, groups, plens)
    table, ptable = widened(table, 4), widened(ptable, 4000)
    want, want_lse = attend(zlib, p, q, table, lens, groups, ptable, plens)
    check(p, q, table, lens, want, want_lse, groups, ptable, plens)
    t, l, g, pt, pl = ints(table), ints(lens), ints(groups), ints(ptable), ints(plens)
    W = (0.05 * torch.randn(d, Hq * hd, generator=p.g, device="cuda")).to(torch.bfloat16)
    n = zlib.zsaa_op_paged_attention_workspace(p.pages, 24, 1, Hq, 2, 4, 4000)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    rows = q.view(24, -1)
    before, after, other = (torch.empty(24, d, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    out = torch.empty_like(q)

    def linear(x, y):
        zlib.zsaa_op_linear(x, W, None, None, y, 24, d, Hq * hd, zlib.ZSAA_BF16, zlib.EPI_STORE)

    def layer():
        linear(rows, before)
        zlib.zsaa_op_paged_attention(p.pages, q, 24, 1, Hq, t, 4, l, g, 2, pt, 4000, pl, out, None, ws, n)
        linear(out.view(24, -1), after)

    layer()
    torch.cuda.synchronize()
    linear(rows, other)
    torch.cuda.synchronize()
    assert torch.equal(before, other) and torch.equal(out, want)
    linear(want.view(24, -1), other)
    torch.cuda.synchronize()
    assert torch.equal(after, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(20):
            layer()
    for _ in range(10):
        out.zero_()
        after.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(after, other)


def test_pages_beyond_32_bit_offsets(zlib):
    """The sequence's pages lie past element 2^31 of the pools."""
    page, Hkv, hd = 256, 8, 128
    n_pages = 2 ** 31 // (page * Hkv * hd) + 40
    k, v = (torch.empty(n_pages, Hkv, page, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pages = zlib.make_pages(k, v)
    T, Hq = 600, 16
    row = [n_pages - 1, n_pages - 2, n_pages - 7]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    qkv = torch.randn(T, (Hq + 2 * Hkv) * hd, generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    q_out = torch.empty(T, Hq, hd, dtype=torch.bfloat16, device="cuda")
    zlib.zsaa_op_paged_append(pages, qkv, qkv.shape[1], zlib.ZSAA_BF16, T, Hq, pos, 1e4, ints([0, T]), 1, ints([row]), 3,
                              ints([T]), q_out)
    small = Pool(zlib, "bf16", Hkv, hd, page, 3)
    small.k.copy_(k[torch.tensor(row[::-1], device="cuda")])
    small.v.copy_(v[torch.tensor(row[::-1], device="cuda")])
    x = np64(qkv).reshape(T, -1, hd)
    kk, _ = small.np()
    want = R.rope(x[:, Hq:Hq + Hkv], np.arange(T)[:, None], 1e4)
    got = R.entries(kk, [2, 1, 0], T).transpose(1, 0, 2)
    assert np.all(np.abs(got - want) <= rope_tol(x[:, Hq:Hq + Hkv], want, True))
    q = q_out[-1:, None].contiguous()
    big = type("P", (), dict(pages=pages))
    out, lse = attend(zlib, big, q, [row], [T])
    check(small, q, [[2, 1, 0]], [T], out, lse)


@pytest.mark.parametrize("cols", [3, 100, 3000])
def test_bad_pages_and_lengths_are_reported(zlib, cols):
    p, q, table, ptable = build(zlib, "bf16", 40, 2, 64, 16, [40, 40], 1, [0, 2], [40])
    table, ptable = widened(table, cols), widened(ptable, cols)
    p.k.nan_to_num_(0.0)
    p.v.nan_to_num_(0.0)
    keep = (p.k.clone(), p.v.clone())

    def reported(call):
        call()
        with pytest.raises(zlib.ZsaaError) as e:
            zlib.zsaa_device_status()
        assert e.value.status == zlib.ZSAA_ERR_INVALID_ARG

    for page in (-1, p.k.shape[0], 2 ** 31 - 1):
        t = [list(r) for r in table]
        t[1][1] = page
        reported(lambda: attend(zlib, p, q, t, [40, 40], [0, 2], ptable, [40]))
        t = [list(r) for r in ptable]
        t[0][2] = page
        reported(lambda: attend(zlib, p, q, table, [40, 40], [0, 2], t, [40]))
        t = [list(r) for r in table]
        t[0][2] = page
        reported(lambda: append_rows(zlib, p, t, [40, 40], [1, 1]))
    reported(lambda: attend(zlib, p, q, [r[:2] for r in table], [40, 30], [0, 2], ptable, [40]))
    reported(lambda: attend(zlib, p, q, table, [40, 40], [0, 2], [r[:2] for r in ptable], [40]))
    reported(lambda: append_rows(zlib, p, [r[:2] for r in table], [33, 30], [1, 1]))
    assert zlib.zsaa_device_status() is None
    for now, then in zip((p.k, p.v), keep):  # the good rows of the reported appends went to entries 39 and 29
        changed = (now != then).any(dim=3).any(dim=1)
        want = torch.zeros_like(changed)
        want[table[1][2], 39 % 16] = want[table[1][1], 29 % 16] = True
        assert torch.equal(changed, want)


@pytest.mark.parametrize("dtype,cols", [("bf16", 4), ("bf16", 100), ("bf16", 5000), ("f32", 4), ("f32", 100)])
@pytest.mark.parametrize("n_q", [1, 4, 16])
def test_negative_lengths_count_as_none(zlib, dtype, cols, n_q):
    lens, plens = [-1, 40, -2 ** 31, 5, -2 ** 31 + n_q, -2 ** 31 + 15], [30, 0]
    p, q, table, ptable = build(zlib, dtype, 40, 2, 64, 16, [max(n, 0) for n in lens], n_q, [0, 3, 6], plens)
    table, ptable = widened(table, cols), widened(ptable, cols)
    out, lse = attend(zlib, p, q, table, lens, [0, 3, 6], ptable, plens)
    check(p, q, table, lens, out, lse, [0, 3, 6], ptable, plens)
    out, lse = attend(zlib, p, q, table, lens)
    check(p, q, table, lens, out, lse)
    out, lse = attend(zlib, p, q, table, lens, [0, 3, 6], ptable, [-2 ** 31, -7])
    check(p, q, table, lens, out, lse)  # (a prefix of a negative length is none)


@pytest.mark.parametrize("rows,pad", [([1, 1, 1], 0), ([1, 1, 1], 1), ([3, 20, 1], 2)])
def test_append_writes_nothing_for_negative_lengths(zlib, rows, pad):
    p = Pool(zlib, "bf16", 2, 64, 16, 9)
    table = [p.row(40, 3, fill=False) for _ in range(3)]
    _, _, q_out = append_rows(zlib, p, table, [-1, -2 ** 31, -2 ** 31 + 7], rows, pad=pad)
    assert (q_out == 7.0).all() and torch.isnan(p.k).all() and torch.isnan(p.v).all()


@pytest.mark.parametrize("dtype,cols", [("bf16", 3), ("bf16", 100), ("bf16", 3000), ("f32", 3), ("f32", 100)])
def test_group_bounds_that_run_backwards_stay_in_bounds(zlib, dtype, cols):
    p, q, table, ptable = build(zlib, dtype, 40, 2, 64, 16, [20] * 4, 1, [0, 4], [40, 40, 40])
    ptable = widened(ptable, cols)
    for groups in ([4, 0, 4, 2], [-5, 9, 1, 4], [2 ** 31 - 1, -2 ** 31, 3, 4], [3, 1, 0, 0]):
        attend(zlib, p, q, table, [20] * 4, groups, ptable, [40, 40, 40])
        try:
            zlib.zsaa_device_status()
        except zlib.ZsaaError as e:
            assert e.status == zlib.ZSAA_ERR_INVALID_ARG


# ------------------------------------------------------------------ append

def rope_tol(x, want, bf16):
    """Products and their sum in float32 from sines and cosines good to 2^-22: of the
    pair's size 4 * 2^-22, then one rounding."""
    h = x.shape[-1] // 2
    pair = np.abs(x[..., :h]) + np.abs(x[..., h:])
    fine = 4 * 2.0 ** -22 * np.concatenate([pair, pair], axis=-1)
    return fine + (R.BF16_HALF if bf16 else R.F32_HALF) * (np.abs(want) + fine)


def append_rows(z, p, table, lens, rows, Hq=4, wide=False, pos=None, pad=0, theta=1e4, seed=9, with_q=True, lead=0):
    """One append of rows[s] new entries per sequence, `lead` rows of padding before and
    `pad` after; returns the call's inputs and q_out (7 where nothing was written)."""
    Hkv, hd = p.k.shape[1], p.k.shape[3]
    T = sum(rows) + pad + lead
    width = (Hq + 2 * Hkv) * hd
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ld = width + 24
    qkv = torch.randn(T, ld, generator=g, device="cuda")
    qkv = qkv if wide or p.k.dtype == torch.float32 else qkv.to(p.k.dtype)
    qkv[:, width:] = float("nan")
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 3 if pos is None else ints(pos)
    q_out = torch.full((T, Hq, hd), 7.0, device="cuda", dtype=p.k.dtype) if with_q else None
    cu = None if all(r == 1 for r in rows) and pad == lead == 0 else ints(lead + np.cumsum([0] + list(rows)))
    z.zsaa_op_paged_append(p.pages, qkv, ld, z.ZSAA_F32 if qkv.dtype == torch.float32 else z.ZSAA_BF16, T, Hq, pos, theta,
                           cu, len(rows), ints(table), len(table[0]), ints(lens), q_out)
    return np64(qkv)[:, :width].reshape(T, -1, hd), pos.cpu().numpy(), q_out


APPENDS = [
    # dtype, Hq, Hkv, hd, page, rows, before (entries in the cache; negative: left padding), wide, pad
    ("bf16", 4, 2, 64, 16, [1], [0], False, 0),
    ("bf16", 8, 8, 128, 16, [1, 1, 1], [15, 16, 130], True, 0),
    ("bf16", 32, 8, 64, 32, [1] * 9, [5] * 9, True, 0),
    ("bf16", 6, 2, 128, 16, [5, 0, 40, 1], [3, 7, 0, 63], False, 3),
    ("bf16", 4, 1, 64, 64, [200, 700, 640], [0, 100, 1], False, 5),
    ("bf16", 3, 1, 128, 16, [4, 4, 4], [-2, 0, -4], True, 0),
    ("f32", 4, 4, 32, 16, [1, 1], [0, 31], True, 0),
    ("f32", 4, 2, 64, 16, [20, 3], [9, 16], True, 2),
    ("f32", 5, 5, 128, 256, [300, 1, 1000], [300, 0, 7], True, 0),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,hd,page,rows,before,wide,pad", APPENDS)
@pytest.mark.parametrize("theta", [10000.0, 500000.0])
def test_append(zlib, dtype, Hq, Hkv, hd, page, rows, before, wide, pad, theta):
    lens = [a + b for a, b in zip(rows, before)]
    cols = max(1, max(-(-n // page) for n in lens)) + 1
    p = Pool(zlib, dtype, Hkv, hd, page, sum(max(0, -(-n // page)) for n in lens) + 2)
    table = [p.row(max(0, n), cols, fill=False) for n in lens]
    lead = 2 if pad else 0
    x, pos, q_out = append_rows(zlib, p, table, lens, rows, Hq, wide, pad=pad, theta=theta, lead=lead)
    k, v = p.np()
    q = np64(q_out)
    bf16 = dtype == "bf16"
    written = np.zeros(k.shape[:3], bool)
    t = lead
    assert np.all(q[:lead] == 7.0)
    for s, n in enumerate(rows):
        for i in range(n):
            e = lens[s] - n + i
            if e < 0:
                assert np.all(q[t] == 7.0)
            else:
                page_no, off = table[s][e // page], e % page
                want = R.rope(x[t, :Hq + Hkv], pos[t], theta)
                tol = rope_tol(x[t, :Hq + Hkv], want, bf16)
                got = np.concatenate([q[t], k[page_no, :, off]])
                assert np.all(np.abs(got - want) <= tol), (s, i)
                value = x[t, Hq + Hkv:]
                assert np.all(np.abs(v[page_no, :, off] - value) <= (R.BF16_HALF * np.abs(value) if bf16 else 0.0))
                written[page_no, :, off] = True
            t += 1
    assert np.all(q[t:] == 7.0)
    assert np.isnan(k[~written]).all() and np.isnan(v[~written]).all(), "an entry that no row owns was written"


def test_append_far_positions_and_no_queries(zlib):
    """Angles of every int32 position: nothing is lost to the size of pos * frequency."""
    pos = [0, 1, 16383, 16384, 1 << 20, (1 << 30) + 12345, 2 ** 31 - 1, -1, -(2 ** 31), 999999999]
    p = Pool(zlib, "f32", 2, 128, 16, 4)
    table = [p.row(len(pos), 2, fill=False)]
    x, _, _ = append_rows(zlib, p, table, [len(pos)], [len(pos)], Hq=4, pos=pos, theta=500000.0, with_q=False)
    k, _ = p.np()
    got = R.entries(k, table[0], len(pos)).transpose(1, 0, 2)
    want = R.rope(x[:, 4:6], np.array(pos)[:, None], 500000.0)
    # the 64-bit reference's own angles are off by a position's size * 2^-52
    slack = 2 * np.abs(x[:, 4:6]).max() * np.abs(np.array(pos, np.float64))[:, None, None] * 2.0 ** -51
    assert np.all(np.abs(got - want) <= rope_tol(x[:, 4:6], want, False) + slack)


def test_append_agrees_with_the_rotation_of_the_projection(zlib):
    """The rotated heads that zsaa_op_linear's epilogue leaves, from the same operands:
    both round the same sums once, from angles that differ in the last bits."""
    T, d, Hq, Hkv, hd = 40, 256, 4, 2, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    A = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
    N = (Hq + 2 * Hkv) * hd
    W = (0.05 * torch.randn(N, d, generator=g, device="cuda")).to(torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 7
    rot, raw = torch.empty(T, N, device="cuda", dtype=torch.bfloat16), torch.empty(T, N, device="cuda")
    zlib.zsaa_op_linear(A, W, None, None, rot, T, N, d, zlib.ZSAA_BF16, zlib.EPI_ROPE, pos=pos,
                        rope_cols=(Hq + Hkv) * hd, rope_hd=hd, rope_theta=10000.0)
    zlib.zsaa_op_linear(A, W, None, None, raw, T, N, d, zlib.ZSAA_BF16, zlib.EPI_STORE_F32)
    p = Pool(zlib, "bf16", Hkv, hd, 16, 4)
    table = [p.row(T, 3, fill=False)]
    q = torch.empty(T, Hq, hd, device="cuda", dtype=torch.bfloat16)
    zlib.zsaa_op_paged_append(p.pages, raw, N, zlib.ZSAA_F32, T, Hq, pos, 10000.0, ints([0, T]), 1, ints(table), 3,
                              ints([T]), q)
    k, v = p.np()
    got = np.concatenate([np64(q), R.entries(k, table[0], T).transpose(1, 0, 2), R.entries(v, table[0], T).transpose(1, 0, 2)], 1)
    want = np64(rot).reshape(T, -1, hd)
    assert np.all(np.abs(got - want) <= 2 * R.BF16_HALF * np.maximum(np.abs(got), np.abs(want)) + 1e-4)
    assert np.mean(got == want) > 0.99
