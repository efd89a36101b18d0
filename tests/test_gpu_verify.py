"""Verification of drafted tokens on the GPU against a plain form in 64 bits, and generation
with drafts over paged caches."""

import numpy as np
import pytest
import torch

import pages_ref as P
import paged_ref as R
from helpers import need_gpu, np64
from test_gpu_paged import DTYPES, attend, ints

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def _gpu(zlib):
    need_gpu()
    yield
    zlib.zsaa_device_status()


def rows(x, dtype, ld, offset):
    """Device rows [a, b, ld] of x [a, b, V], `offset` elements into a buffer of NaNs, and
    their values in 64 bits."""
    a, b, V = x.shape
    buf = torch.full((offset + a * b * ld + 8,), NAN, device="cuda", dtype=DTYPES[dtype])
    t = buf[offset:offset + a * b * ld]
    t.view(a * b, ld)[:, :V] = torch.from_numpy(x.reshape(a * b, V)).cuda().to(DTYPES[dtype])
    return t, np64(t).reshape(a, b, ld)[:, :, :V]


def call(z, target, draft, drafts, temp, uniform, dtype="f32", pad=0, offset=0, lens=None):
    """NumPy in, NumPy out, and the target and draft rows as stored."""
    S, n1, V = target.shape
    n, ld = n1 - 1, V + pad
    t, t64 = rows(target, dtype, ld, offset)
    d, d64 = rows(draft, dtype, ld, offset + 1) if draft is not None and n else (None, None)
    ws = torch.full((z.zsaa_op_draft_verify_workspace(S, n, V),), 255, dtype=torch.uint8, device="cuda")
    acc, tok = (torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((S,), (S, n1)))
    logp = torch.full((S, n1), 7.0, device="cuda")
    f32 = lambda x: None if x is None else torch.from_numpy(np.asarray(x, np.float32)).cuda()
    lens = np.arange(S) + 20 if lens is None else lens
    lens_out = ints(np.zeros(S))
    z.zsaa_op_draft_verify(t, ld, d, ld, z.ZSAA_F32 if dtype == "f32" else z.ZSAA_BF16, S, n, V, ints(drafts) if n else None,
                           f32(temp), f32(uniform), acc, tok, logp, ints(lens), lens_out, ws, ws.numel())
    acc, tok = acc.cpu().numpy(), tok.cpu().numpy()
    np.testing.assert_array_equal(lens_out.cpu().numpy(), np.maximum(lens - n + acc, 0))
    return acc, tok, logp.cpu().numpy(), t64, d64


def check(z, target, draft, drafts, temp, uniform, **kw):
    acc, tok, logp, t64, d64 = call(z, target, draft, drafts, temp, uniform, **kw)
    want_acc, want, want_logp, near, border = P.verify(t64, d64, drafts, temp, uniform)
    # a row's sum is off by at most 2^-22 (an exponential) + 2^-23 of the exponents' mean size (two
    # roundings, 19 or less over 2^17 tokens) + 32 2^-24 (the additions): below 2^-17; a decision by
    # two of them.  The sums that pick a token are good to 2^-36 of the sums of p and q.
    assert near > 2.0 ** -16 and border > 2.0 ** -34, "a decision is too near to be told: %g %g" % (near, border)
    np.testing.assert_array_equal(acc, want_acc)
    np.testing.assert_array_equal(tok, want)
    assert np.all(np.abs(logp - want_logp) <= 2.0 ** -17 + R.F32_HALF * np.abs(want_logp)), np.abs(logp - want_logp).max()


def draw(S, n, V, seed, banned=0.0, noise=0.8, temp=None):
    """Logits, drafts that follow the draft rows, and numbers."""
    r = np.random.default_rng(seed)
    target = (3 * r.standard_normal((S, n + 1, V))).astype(np.float32)
    draft = (target[:, :n] + noise * r.standard_normal((S, n, V))).astype(np.float32)
    if banned:
        out = r.random((S, 1, V)) < banned
        out[:, :, V // 2] = False
        target[np.broadcast_to(out, target.shape)] = -INF
        draft[np.broadcast_to(out, draft.shape)] = -INF
    t = np.ones(S) if temp is None else np.maximum(np.asarray(temp, np.float64), 1e-3)
    drafts = np.argmax(draft / t[:, None, None] + r.gumbel(size=draft.shape), axis=2)
    return target, draft, drafts, r.random((S, n + 1)).astype(np.float32), r


@pytest.mark.parametrize("dtype,pad,offset", [("f32", 0, 0), ("f32", 3, 1), ("bf16", 0, 0), ("bf16", 5, 3)])
@pytest.mark.parametrize("S,n,V", [(1, 4, 128256), (5, 1, 1000), (3, 15, 777), (40, 3, 50), (2, 2, 8193), (7, 0, 8192),
                                   (9, 5, 16385), (1, 0, 1), (3, 2, 1), (33, 2, 7), (2, 7, 40001), (300, 1, 33)])
def test_verify(zlib, S, n, V, dtype, pad, offset):
    target, draft, drafts, u, _ = draw(S, n, V, S + n + V)
    check(zlib, target, draft, drafts, None, u, dtype=dtype, pad=pad, offset=offset)
    check(zlib, target, None, drafts, None, u, dtype=dtype, pad=pad, offset=offset)


@pytest.mark.parametrize("lookup", [False, True])
@pytest.mark.parametrize("S,n,V,dtype", [(700, 5, 60, "f32"), (5000, 1, 9, "bf16"), (400, 15, 1000, "f32"), (45, 4, 131072, "bf16"),
                                         (40, 4, 140001, "f32")])
def test_verify_large_calls(zlib, S, n, V, dtype, lookup):
    """Calls that scan a draft's rows of all sequences before the next draft's, with every kind
    of end: a draft refused, none left, a row without a distribution, a temperature of 0."""
    temp = np.random.default_rng(1).choice([0.0, 0.7, 1.0, 1.4], S)
    temp[S // 2] = -1.0
    target, draft, drafts, u, r = draw(S, n, V, S + V, noise=0.5, temp=temp)
    drafts = np.where(np.arange(n) < r.integers(0, n + 2, (S, 1)), drafts, -1)
    for s in range(0, S, 7):
        target[s, r.integers(0, n + 1), r.integers(0, V)] = (NAN, INF)[s % 2]
    for s in range(3, S, 7):
        draft[s, r.integers(0, n), r.integers(0, V)] = NAN
    check(zlib, target, None if lookup else draft, drafts, temp, u, dtype=dtype, pad=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_verify_temperatures_bans_and_early_ends(zlib, dtype):
    temp = np.array([0, 0.05, 0.3, 0.7, 1.0, 1.5, 4.0, 60.0, 1e4, 0.0, 1.0, 2.0 ** -30, 2.0 ** -70, 2.0 ** 40], np.float32)
    S = len(temp)
    target, draft, drafts, u, r = draw(S, 4, 5000, 3, banned=0.5, temp=temp)
    check(zlib, target, draft, drafts, temp, u, dtype=dtype)
    check(zlib, target, None, drafts, temp, u, dtype=dtype)
    ended = np.where(np.arange(4) < r.integers(0, 5, (S, 1)), drafts, -1)
    ended[3, 0], ended[4, 2], ended[5, 1] = 5000, -2 ** 31, 2 ** 31 - 1
    check(zlib, target, draft, ended, temp, u, dtype=dtype)


@pytest.mark.parametrize("draft_rows", [False, True])
def test_verify_rows_without_a_distribution(zlib, draft_rows):
    """NaN, +inf and all -inf in a target or a draft row, at the first, a middle and the last."""
    target, draft, drafts, u, _ = draw(12, 3, 3000, 8, noise=0.05)  # (nearly all drafts stand)
    x = draft if draft_rows else target
    for s in range(9):
        j = s % 3 if draft_rows else (0, 1, 3)[s % 3]
        x[s, j, (0, 1777, 2999)[s // 3]] = (NAN, INF, NAN)[s // 3]
    x[9, 1], x[10, 0], x[11, 2] = -INF, -INF, NAN
    check(zlib, target, draft, drafts, None, u)
    check(zlib, target, draft, drafts, np.where(np.arange(12) % 2, 0.0, 0.9), u)


@pytest.mark.parametrize("t", [-1.0, NAN, INF, -INF, 2.0 ** 65, -0.0])
def test_verify_temperatures_out_of_range(zlib, t):
    target, draft, drafts, u, _ = draw(3, 2, 900, 4)
    temp = np.array([1, t, 0.5])
    check(zlib, target, draft, drafts, temp, u)
    if t != 0:
        assert call(zlib, target, draft, drafts, temp, u)[1][1].tolist() == [-1, -1, -1]


def test_verify_numbers_at_and_beyond_their_ends(zlib):
    target, draft, drafts, u, _ = draw(8, 2, 2000, 5)
    for v in (0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, INF, -INF, NAN):
        u[:, 2] = v
        check(zlib, target, draft, drafts, None, u)
    for v in (0.0, 2.0, -1.0, NAN):
        u[:, :2] = v
        check(zlib, target, draft, drafts, None, u)


@pytest.mark.parametrize("S", [5, 1700])  # (the second scans draft by draft)
@pytest.mark.parametrize("lookup", [False, True])
@pytest.mark.parametrize("gap,t", [(800.0, 1.0), (40.0, 0.05), (1e30, 1.0), (90.0, 1.0)])
def test_verify_the_number_0_takes_every_draft_that_is_possible(zlib, gap, t, lookup, S):
    """u q(x) < p(x) is 0 < p(x) then, also where p(x) is e^-800 or smaller; a banned token has 0."""
    V, x = 50, 5
    target = np.zeros((S, 2, V), np.float32)
    target[:, :, 7] = gap
    draft = np.zeros((S, 1, V), np.float32)
    draft[:, :, x] = gap
    target[3, 0, x] = -INF
    for v in (0.0, -1.0, NAN, 1e-45):
        u = np.full((S, 2), 0.5, np.float32)
        u[:, 0] = v
        acc, tok, logp, _, _ = call(zlib, target, None if lookup else draft, np.full((S, 1), x), np.full(S, t), u)
        # (1e-45 is e^-103.3: it refuses what is less likely than that)
        stands = np.arange(S) != 3 if v != 1e-45 or gap == 90.0 else np.zeros(S, bool)
        np.testing.assert_array_equal(acc, stands)
        np.testing.assert_array_equal(tok, np.where(stands[:, None], [x, 7], [7, -1]))
        want = -gap / float(np.float32(t))  # (as in check)
        assert np.all(np.abs(logp[stands] - [want, 0.0]) <= 2.0 ** -17 + R.F32_HALF * abs(want))


def test_verify_equal_rows_stand_and_opposite_ones_do_not(zlib):
    target, _, _, u, r = draw(6, 3, 4000, 6)
    drafts = np.argmax(target[:, :3] + r.gumbel(size=(6, 3, 4000)), 2)
    acc, tok, _, _, _ = call(zlib, target, target[:, :3].copy(), drafts, None, u)
    assert (acc == 3).all()
    # a draft row on other tokens than the target's: nothing of p is taken off
    draft = np.full((6, 3, 4000), -INF, np.float32)
    draft[:, :, 2000:] = 0
    target[:, :, 2000:] = -INF
    drafts = r.integers(2000, 4000, (6, 3))
    check(zlib, target, draft, drafts, None, u)
    # a token that the draft row calls impossible and the target does not stands
    drafts = r.integers(0, 2000, (6, 3))
    acc, _, _, _, _ = call(zlib, target, draft, drafts, None, u)
    assert (acc == 3).all()
    # all of the target on the refused token (q is nearly 1 there): what is left of p is 0
    target[:], draft[:] = -INF, -INF
    target[:, :, 7], draft[:, :, 7] = 0, 0
    u[:] = 1.0
    acc, tok, _, _, _ = call(zlib, target, None, np.full((6, 3), 7), None, u)
    assert (acc == 3).all() and (tok == 7).all()


@pytest.mark.parametrize("S,V", [(2000, 14), (400, 100), (500, 1000), (60, 20000), (12, 128256)])
@pytest.mark.parametrize("differ", ["nowhere", "in one", "in the largest"])
def test_verify_draft_rows_that_agree_with_the_targets(zlib, differ, S, V):
    """A banned draft over rows that are equal leaves nothing of p - q: the token is drawn from p.  One
    logit apart by little, it leaves a residual of 1e-9 and more, of which every token has a part."""
    r = np.random.default_rng(V)
    target = (2 * r.standard_normal((S, 2, V))).astype(np.float32)
    drafts, seq = r.integers(0, V, (S, 1)), np.arange(S)
    target[seq, :, drafts[:, 0]] = -INF
    draft = target[:, :1].copy()
    if differ != "nowhere":
        i = (drafts[:, 0] + 1) % V if differ == "in one" else draft[:, 0].argmax(1)
        draft[seq, 0, i] += (10 ** r.uniform(-7, -1, S)).astype(np.float32)
    u = r.random((S, 2)).astype(np.float32)
    acc, tok, logp, t64, d64 = call(zlib, target, draft, drafts, None, u, pad=1)  # (rows of both kinds start anywhere in 16 bytes)
    assert (acc == 0).all() and (logp > -INF).all()
    told = 0
    for s in range(S):
        _, want, _, _, border = P.verify(t64[s:s + 1], d64[s:s + 1], drafts[s:s + 1], None, u[s:s + 1])
        if border > 2.0 ** -34:
            told += 1
            assert tok[s, 0] == want[0, 0], (s, border)
    assert told > 0 or (differ != "nowhere" and V > 20000)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_verify_greedy_takes_the_first_of_equal_logits(zlib, dtype):
    target = np.zeros((4, 3, 20000), np.float32)
    target[0, 0, [9000, 17000]] = 1
    target[0, 1, 19999] = 1
    target[1] = -0.0
    target[2, :, 5::7] = 2.5
    target[3] = -INF
    target[3, :, 12345] = -1e30
    drafts = np.array([[9000, 5], [0, 0], [5, 12], [12345, 12345]])
    u = np.random.default_rng(0).random((4, 3)).astype(np.float32)
    check(zlib, target, target[:, :2].copy(), drafts, np.zeros(4), u, dtype=dtype)
    assert call(zlib, target, None, drafts, np.zeros(4), u, dtype=dtype)[1].tolist() == [
        [9000, 19999, -1], [0, 0, 0], [5, 5, -1], [12345, 12345, 12345]]


@pytest.mark.parametrize("level", [-3e4, 1e4, 1e6, -1e7, 3e7, 1e9, -1e12, 1e30, -1e30, 3e38])
def test_verify_logits_of_any_size(zlib, level):
    target, draft, drafts, u, _ = draw(6, 2, 3001, 7)
    for x in (target, draft):
        x[0] = (x[0] + np.float32(level)).astype(np.float32)
        x[1, :, 3000] = np.float32(level)
        x[2, :, :] = np.float32(level)
        x[3, :, ::2] = np.float32(level)
        x[4] *= np.float32(min(abs(level), 1e36))
    # (a level that all share makes near decisions: the numbers decide clearly there)
    u[:, :2] = np.where(np.arange(6)[:, None] % 2, 0.02, 0.5)
    acc, tok, logp, t64, d64 = call(zlib, target, draft, drafts, None, u)
    want_acc, want, want_logp, near, border = P.verify(t64, d64, drafts, None, u)
    assert near > 2.0 ** -16 and border > 2.0 ** -34
    np.testing.assert_array_equal(acc, want_acc)
    np.testing.assert_array_equal(tok, want)
    assert np.all(np.abs(logp - want_logp) <= 2.0 ** -17 + R.F32_HALF * np.abs(want_logp))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_verify_long_rows(zlib, dtype):
    """More stretches and groups than a warp and a CTA hold at once."""
    for S, n in ((1, 1), (2, 0)):
        target, draft, drafts, u, _ = draw(S, n, 3000001, 13)
        check(zlib, target, draft, drafts, None, u, dtype=dtype, offset=1)
        check(zlib, target, None, drafts, np.zeros(S), u, dtype=dtype, offset=1)


@pytest.mark.parametrize("spread", [0.0, 0.3, 3.0])
@pytest.mark.parametrize("with_draft", [False, True])
def test_verify_picks_tokens_as_64_bits_do(zlib, spread, with_draft):
    """Borders 2^-17 apart: sums of float32 terms would pick another token now and then."""
    r = np.random.default_rng(11)
    S, V = 150, 128256
    target = (spread * r.standard_normal((S, 1 + with_draft, V))).astype(np.float32)
    u = r.random((S, 1 + with_draft)).astype(np.float32)
    if not with_draft:
        return check(zlib, target, None, np.zeros((S, 0)), None, u)
    draft = (target[:, :1] + r.standard_normal((S, 1, V))).astype(np.float32)
    u[:, 0] = 0.999
    check(zlib, target, draft, np.argmax(draft, 2), None, u)


def test_verify_the_same_bits_again_and_without_the_optional_outputs(zlib):
    z, S, n, V = zlib, 20, 4, 30000
    target, draft, drafts, u, _ = draw(S, n, V, 9)
    first, again = (call(z, target, draft, drafts, None, u) for _ in range(2))
    for a, b in zip(first[:3], again[:3]):
        np.testing.assert_array_equal(a, b)
    t, d = torch.from_numpy(target).cuda(), torch.from_numpy(draft).cuda()
    ws = torch.empty(z.zsaa_op_draft_verify_workspace(S, n, V), dtype=torch.uint8, device="cuda")
    acc, tok = ints(np.zeros(S)), ints(np.zeros((S, n + 1)))
    z.zsaa_op_draft_verify(t, V, d, V, z.ZSAA_F32, S, n, V, ints(drafts), None, torch.from_numpy(u).cuda(), acc, tok, None, None,
                           None, ws, ws.numel())
    np.testing.assert_array_equal(tok.cpu().numpy(), first[1])


def test_verify_rows_far_apart_and_draft_rows_of_another_stride(zlib):
    """Element offsets past 2^31, and draft rows closer together than the target's."""
    z, S, n, V, ld, draft_ld = zlib, 3, 1, 1000, 1 << 29, 1003
    target, draft, drafts, u, _ = draw(S, n, V, 3)
    t = torch.empty((S * (n + 1) - 1) * ld + V, device="cuda")
    for i, row in enumerate(target.reshape(-1, V)):
        t[i * ld:i * ld + V] = torch.from_numpy(row).cuda()
    d = torch.full((S * n, draft_ld), NAN, device="cuda")
    d[:, :V] = torch.from_numpy(draft.reshape(-1, V)).cuda()
    want = P.verify(target.astype(np.float64), draft.astype(np.float64), drafts, None, u)
    assert want[3] > 2.0 ** -16 and want[4] > 2.0 ** -34
    ws = torch.empty(z.zsaa_op_draft_verify_workspace(S, n, V), dtype=torch.uint8, device="cuda")
    acc, tok = ints(np.zeros(S)), ints(np.zeros((S, n + 1)))
    z.zsaa_op_draft_verify(t, ld, d, draft_ld, z.ZSAA_F32, S, n, V, ints(drafts), None, torch.from_numpy(u).cuda(), acc, tok, None,
                           None, None, ws, ws.numel())
    np.testing.assert_array_equal(tok.cpu().numpy(), want[1])


def test_verify_lengths_in_place_and_graphs_on_two_streams(zlib):
    z, S, n, V = zlib, 3, 2, 9000
    runs = []
    for seed in (1, 2):
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            target, draft, drafts, u, _ = draw(S, n, V, seed)
            st = dict(t=torch.from_numpy(target).cuda(), d=torch.from_numpy(draft).cuda(), x=ints(drafts),
                      u=torch.from_numpy(u).cuda(), acc=ints(np.zeros(S)), tok=ints(np.zeros((S, n + 1))), lens=ints([9, 1, 50]),
                      ws=torch.empty(z.zsaa_op_draft_verify_workspace(S, n, V), dtype=torch.uint8, device="cuda"))

            def go(st=st):
                z.zsaa_op_draft_verify(st["t"], V, st["d"], V, z.ZSAA_F32, S, n, V, st["x"], None, st["u"], st["acc"], st["tok"],
                                       None, st["lens"], st["lens"], st["ws"], st["ws"].numel())
            go()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                go()
        runs.append((side, graph, st))
    want = []
    for (side, graph, st), seed in zip(runs, (11, 12)):
        target, draft, drafts, u, _ = draw(S, n, V, seed)
        st["t"].copy_(torch.from_numpy(target))
        st["d"].copy_(torch.from_numpy(draft))
        st["x"].copy_(ints(drafts))
        st["u"].copy_(torch.from_numpy(u))
        st["lens"].copy_(ints([9, 1, 50]))
        want.append(P.verify(target.astype(np.float64), draft.astype(np.float64), drafts, None, u))
        assert want[-1][3] > 2.0 ** -16 and want[-1][4] > 2.0 ** -34
    torch.cuda.synchronize()
    for side, graph, _ in runs:
        with torch.cuda.stream(side):
            graph.replay()
    torch.cuda.synchronize()
    for (_, _, st), w in zip(runs, want):
        np.testing.assert_array_equal(st["tok"].cpu().numpy(), w[1])
        np.testing.assert_array_equal(st["lens"].cpu().numpy(), np.maximum(np.array([9, 1, 50]) - n + w[0], 0))


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_generation_with_drafts_over_counted_pages(zlib, dtype):
    """Two prompts become three samples each; every step takes pages, appends a token and
    three drafts of a model without layers, attends, verifies and gives pages back, lengths
    on the device throughout.  The logits are those of the whole texts without a cache, and
    the tokens those that the logits at hand ask for."""
    from test_gpu_beam import Search
    z, m, page, n, kids = zlib, Search(zlib, dtype), 16, 3, 3
    rng = np.random.default_rng(2)
    prompts = [list(rng.integers(0, m.V, k)) for k in (37, 32)]
    S, cols, n_pages = len(prompts) * kids, 6, 40
    ks, vs = ([torch.full((n_pages, m.Hkv, page, m.hd), NAN, device="cuda", dtype=m.dt) for _ in range(m.L)] for _ in range(2))
    layers = z.make_pages_list(ks, vs)

    class Pool:
        def __init__(self, l):
            self.pages = layers[l]

    pool = [Pool(l) for l in range(m.L)]
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    new = lambda *size: torch.full(size, -1, dtype=torch.int32, device="cuda")

    def forward(tokens, pos, cu, table, lens, rows):
        """One call of all layers over rows of `rows` tokens per sequence."""
        x = m.embed[tokens.view(-1).long()]
        for l in range(m.L):
            x = m.layer(l, x, pos, pool[l], cu, table.shape[0], table, lens, lambda q: attend(
                z, pool[l], q.view(table.shape[0], rows, m.Hq, m.hd), table.tolist(), lens.tolist())[0])
        return x

    # the prompts but for their last tokens, 8 tokens at a time
    table, lens = new(2, cols), ints([0, 0])
    got = ints([0, 0])
    z.zsaa_op_paged_resize(refs, n_pages, page, 2, table, cols, lens, ints([len(p) - 1 for p in prompts]), got)
    for b, prompt in enumerate(prompts):
        for at in range(0, len(prompt) - 1, 8):
            part = prompt[at:min(at + 8, len(prompt) - 1)]
            forward(ints(part), ints(np.arange(at, at + len(part))), ints([0, len(part)]), table[b:b + 1].contiguous(),
                    ints([at + len(part)]), len(part))
    kid_table, lens = new(S, cols), new(S)
    z.zsaa_op_paged_fork(layers, refs, 2, table, cols, got, S, ints([0, 0, 0, 1, 1, 1]), None, kid_table, lens)
    z.zsaa_op_paged_resize(refs, n_pages, page, 2, table, cols, got, ints([0, 0]), ints([0, 0]))  # the prompts' own rows end
    table = kid_table
    texts = [list(prompts[s // kids]) for s in range(S)]
    temp = np.array([0.0, 0.8, 1.3] * 2, np.float32)
    d_temp = torch.from_numpy(temp).cuda()
    ws = torch.empty(z.zsaa_op_draft_verify_workspace(S, n, m.V), dtype=torch.uint8, device="cuda")
    for step in range(6):
        # drafts: the model without its layers, one token after the other
        tok = [ints([t[-1] for t in texts])]
        draft = []
        for j in range(n):
            draft.append(m.linear(m.embed[tok[-1].long()], m.head, z.EPI_STORE_F32, torch.float32))
            noise = torch.from_numpy(rng.gumbel(size=(S, m.V)).astype(np.float32)).cuda()
            tok.append(torch.argmax(draft[-1] + d_temp[:, None] * noise, 1).to(torch.int32))
        tokens, draft = torch.stack(tok, 1).contiguous(), torch.stack(draft, 1).contiguous()
        want_lens, held = lens + (n + 1), new(S)
        z.zsaa_op_paged_resize(refs, n_pages, page, S, table, cols, lens, want_lens, held)
        assert torch.equal(held, want_lens)
        pos = (lens[:, None] + torch.arange(n + 1, device="cuda", dtype=torch.int32)).reshape(-1).contiguous()
        x = forward(tokens, pos, ints(np.arange(S + 1) * (n + 1)), table, held, n + 1)
        logits = m.linear(x.contiguous(), m.head, z.EPI_STORE_F32, torch.float32).view(S, n + 1, m.V)
        u = rng.random((S, n + 1)).astype(np.float32)
        acc, out, kept = new(S), new(S, n + 1), new(S)
        z.zsaa_op_draft_verify(logits, m.V, draft, m.V, z.ZSAA_F32, S, n, m.V, tokens[:, 1:].contiguous(), d_temp,
                               torch.from_numpy(u).cuda(), acc, out, None, held, kept, ws, ws.numel())
        lens = new(S)
        z.zsaa_op_paged_resize(refs, n_pages, page, S, table, cols, held, kept, lens)
        assert torch.equal(lens, kept)
        w_acc, w_out, _, near, border = P.verify(np64(logits), np64(draft), tokens[:, 1:].cpu().numpy(), temp, u)
        assert near > 2.0 ** -16 and border > 2.0 ** -34
        np.testing.assert_array_equal(out.cpu().numpy(), w_out)
        np.testing.assert_array_equal(acc.cpu().numpy(), w_acc)
        for s in range(S):
            texts[s] += [int(t) for t in w_out[s] if t >= 0]
            assert lens[s].item() == len(texts[s]) - 1
            ref, row = m.reference(texts[s][:-1]), np64(logits[s, w_acc[s]])
            if dtype == "f32":
                assert np.abs(row - ref).max() <= 1e-4 * np.abs(ref).max(), (step, s)
            else:
                assert np.linalg.norm(row - ref) / np.linalg.norm(ref) <= 2e-2, (step, s)
        used = set()
        for s in range(S):
            used |= set(table[s, :-(-lens[s].item() // page)].tolist())
        assert (refs > 0).sum().item() == len(used) and refs.sum().item() == sum(-(-x // page) for x in lens.tolist())
    z.zsaa_op_paged_resize(refs, n_pages, page, S, table, cols, lens, ints([0] * S), new(S))
    assert refs.abs().sum().item() == 0
