"""Selection of continuations and reordering of page tables on the GPU, against plain
64-bit forms; and a whole beam search over paged caches."""

import numpy as np
import pytest
import torch

import paged_ref as R
from helpers import need_gpu, np64
from test_gpu_paged import Pool, attend, ints

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(autouse=True)
def _gpu(zlib):
    need_gpu()
    yield
    zlib.zsaa_device_status()


def select(z, logits, scores, done, eos, K, ld=None, offset=0):
    """logits [B, W, V] NumPy; the rows lie `offset` floats into a buffer, `ld` apart."""
    B, W, V = logits.shape
    ld = V if ld is None else ld
    buf = torch.full((offset + B * W * ld,), NAN, device="cuda")
    rows = buf[offset:].view(B * W, ld)
    rows[:, :V] = torch.from_numpy(logits.reshape(B * W, V)).cuda()
    n = z.zsaa_op_beam_select_workspace(B, W, V, K)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    s_out = torch.full((B, K), 7.0, device="cuda")
    parent, token = (torch.full((B, K), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    d_out = torch.full((B, K), 9, dtype=torch.uint8, device="cuda")
    z.zsaa_op_beam_select(rows, ld, B, W, V, None if scores is None else torch.from_numpy(scores).cuda(),
                          None if done is None else torch.from_numpy(done.astype(np.uint8)).cuda(), eos, K, s_out, parent,
                          token, d_out, ws, n)
    return [t.cpu().numpy() for t in (s_out, parent, token, d_out)]


def check_select(z, logits, scores, done, eos, K, **kw):
    want = R.select(logits, scores, done, eos, K)
    # continuations of two beams must not be closer than the error of the totals allows
    assert want[4] > 2e-6, "two totals are too close to be told apart: %g" % want[4]
    got = select(z, logits, scores, done, eos, K, **kw)
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[2], want[2])
    np.testing.assert_array_equal(got[3], want[3])
    fin = np.isfinite(want[0])
    np.testing.assert_array_equal(got[0][~fin], want[0][~fin].astype(np.float32))
    # lse: the sum's terms to 2^-22 each, their 32 additions to 2^-20; then one rounding
    assert np.all(np.abs(got[0][fin] - want[0][fin]) <= 2.0 ** -19 + R.F32_HALF * np.abs(want[0][fin]))


def draw(B, W, V, seed, scale=3.0):
    r = np.random.default_rng(seed)
    return (scale * r.standard_normal((B, W, V))).astype(np.float32), (-20 * r.random((B, W))).astype(np.float32), r


@pytest.mark.parametrize("B,W,V,K", [
    (1, 1, 1, 1), (1, 1, 3, 3), (2, 3, 2, 6), (1, 4, 1000, 8), (3, 5, 2047, 5), (2, 8, 2049, 16), (1, 1, 40001, 64),
    (1, 64, 333, 64), (5, 2, 8192, 4), (1, 4, 128256, 8), (4, 2, 50257, 2), (90, 4, 8193, 3), (1, 3, 8188, 64),
    (1, 1, 600001, 64), (1, 12, 300000, 20), (2, 16, 5000, 32), (3, 9, 700, 64), (30, 16, 4100, 8), (1, 32, 20000, 33)])
def test_select(zlib, B, W, V, K):
    logits, scores, _ = draw(B, W, V, B + W + V + K)
    check_select(zlib, logits, scores, None, -1, K)
    check_select(zlib, logits, None, None, 0, K)


@pytest.mark.parametrize("offset,ld", [(0, 5003), (1, 5001), (2, 5002), (3, 5000), (1, 5007)])
def test_select_rows_at_any_alignment(zlib, offset, ld):
    logits, scores, _ = draw(2, 3, 5000, 11)
    check_select(zlib, logits, scores, None, -1, 7, ld=ld, offset=offset)


@pytest.mark.parametrize("K", [1, 6, 64])
def test_select_masks_ended_beams_and_what_is_not_finite(zlib, K):
    logits, scores, r = draw(8, 6, 3000, 5)
    done = r.random((8, 6)) < 0.3
    logits[r.random(logits.shape) < 0.5] = -INF
    logits[0, 2] = -INF                       # nothing allowed
    logits[1, :, 5:] = -INF                   # a grammar leaves five tokens
    logits[2, 1, 77] = NAN
    logits[3, 0, 2999] = INF
    logits[4, 3] = NAN
    scores[5] = [0, -INF, -INF, -INF, -INF, -INF]  # the first step of a search
    scores[6, 2] = NAN
    done[6] = True
    scores[7] = -INF
    check_select(zlib, logits, scores, done, 2, K)
    check_select(zlib, logits, scores, None, 2, K)


def test_select_ties(zlib):
    logits = np.zeros((3, 4, 9000), np.float32)
    logits[1] = -0.0
    logits[1, :, ::2] = 0.0
    logits[2, :, 4000:] = 2.5
    for K in (1, 9, 64):
        check_select(zlib, logits, None, None, -1, K)
    scores = np.array([[0, 0, 0, 0], [-1, 0, -1, 0], [-2, -2, -1, -1]], np.float32)
    check_select(zlib, logits, scores, None, -1, 20)


def test_select_values_that_crowd_one_warp(zlib):
    """Descending logits put the best values into neighbouring places, and stretches of a
    few very large ones into one warp's: more than the candidate list holds."""
    V = 16384
    down = -np.arange(V, dtype=np.float32) * 1e-3
    crowd = np.zeros(V, np.float32)
    at = (np.arange(V) % 1024) < 128  # one warp of eight, whatever the chunk
    crowd[at] = 10 + np.arange(at.sum()) * 1e-3
    logits = np.stack([down, crowd, down[::-1], crowd[::-1]])[:, None]
    for K in (1, 8, 33, 64):
        check_select(zlib, np.ascontiguousarray(logits), None, None, -1, K)
    many = np.ascontiguousarray(np.repeat(logits, 90, axis=0))  # enough rows for the long chunks
    check_select(zlib, many, None, None, -1, 64)


def test_select_long_rows_with_the_best_in_few_stretches(zlib):
    """Lists of more than 63 stretches are merged in rounds; the best values lie in the
    first stretch, in the last, and in one of the second round."""
    V = 600000
    logits = np.full((3, 1, V), -30, np.float32) + (np.arange(V) % 977).astype(np.float32) * 1e-4
    best = np.arange(200, dtype=np.float32) * 1e-2
    logits[0, 0, 17:217] = best
    logits[1, 0, -200:] = -best
    logits[2, 0, 400000:400200] = best[::-1]
    for row in logits:  # (one row: as many stretches as there are)
        for K in (1, 9, 64):
            check_select(zlib, row[None], None, None, -1, K)


def test_select_many_beams_some_ended(zlib):
    logits, scores, r = draw(3, 20, 4000, 21)
    done = r.random((3, 20)) < 0.4
    done[1, 8:] = True
    logits[2, 11] = -INF
    for K in (5, 30):
        check_select(zlib, logits, scores, done, 3, K)


@pytest.mark.parametrize("level", [-3e4, 1e4, 80.0])
def test_select_logits_far_from_zero(zlib, level):
    """x - max first: the totals do not lose what the common level is."""
    logits, scores, _ = draw(2, 4, 3001, 8)
    logits = (np.round(logits * 256) / 256 + level).astype(np.float32)
    check_select(zlib, logits, scores, None, -1, 8)


def ulps(level, steps):
    """float32 numbers `steps` units of the last place above `level`."""
    x = np.float32(level)
    return x + np.asarray(steps, np.float32) * np.spacing(np.abs(x))


def check_levels(z, logits, scores, K):
    """As check_select, with totals that take the maximum off first, so that 64 bits hold
    what they are at any level: score + ((x - max) - log sum exp(x - max))."""
    B, W, V = logits.shape
    top = logits.max(-1, keepdims=True).astype(np.float64)
    gap = logits - top
    total = scores[..., None] + (gap - np.log(np.exp(gap).sum(-1, keepdims=True)))
    want = []
    for b in range(B):
        w, v = np.meshgrid(np.arange(W), np.arange(V), indexing="ij")
        order = np.lexsort((v.ravel(), -logits[b].ravel().astype(np.float64), w.ravel(), -total[b].ravel()))[:K + 1]
        t, w, v = total[b].ravel()[order], w.ravel()[order], v.ravel()[order]
        apart = (t[:-1] - t[1:])[(w[:-1] != w[1:]) & (t[:-1] != t[1:])]
        assert apart.size == 0 or apart.min() > 2e-6, "two totals are too close to be told apart"
        want.append((t[:K], w[:K], v[:K]))
    got = select(z, logits, scores, None, -1, K)
    for b, (t, w, v) in enumerate(want):
        np.testing.assert_array_equal(got[1][b], w)
        np.testing.assert_array_equal(got[2][b], v)
        # as in check_select
        assert np.all(np.abs(got[0][b] - t) <= 2.0 ** -19 + R.F32_HALF * np.abs(t)), (got[0][b], t)


@pytest.mark.parametrize("V", [4096, 70001])
@pytest.mark.parametrize("level", [1e6, -1e6, 1e7, -1e7, 3e7, -3e7, 1e8, -1e8, 1e9, -1.5e9, 1e10, -1e10, 1e12, -1e12, 1e30,
                                   -1e30, 3e38, -3e38])
def test_select_logits_of_any_size(zlib, level, V):
    """Rows far from zero as a whole or in part: masks of a large finite number, forced
    tokens, values a few units of the last place apart."""
    ordinary, scores, r = draw(5, 3, V, 17)
    logits = ordinary.copy()
    logits[0] = ulps(level, r.integers(-3, 4, (3, V)))   # all beams
    logits[1, 0] = np.float32(level)                     # one beam, all of it the same
    logits[2, :, V - 2] = ulps(level, [0, 1, 2])         # one token in the last stretch
    logits[3, :, 5] = ulps(level, [2, 0, 1])             # one in the first
    keep = r.permutation(V)[:5]                          # all but five
    logits[4] = np.float32(level)
    logits[4][:, keep] = ordinary[4][:, keep]
    for K in (1, 8, 64):
        check_levels(zlib, logits, scores, K)


@pytest.mark.parametrize("low,high", [(0.9 * 2.0 ** 100, 2.0 ** 100), (-(2.0 ** 100), -0.9 * 2.0 ** 100), (2.0 ** 23 - 1, 2.0 ** 23 + 1),
                                      (1.0, 2.0 ** 100), (-(2.0 ** 100), 1.0), (-30.0, 9.5), (-41.0, 0.0), (-80.0, 7.0)])
def test_select_maxima_of_different_warps_and_stretches(zlib, low, high):
    """Warps and stretches whose own maxima lie far below the row's, or next to it."""
    V = 50000
    logits, scores, r = draw(4, 2, V, 23, scale=0.5)
    at = np.arange(V)
    logits[0] = np.where((at % 1024) // 128 == 3, np.float32(high), np.float32(low))  # one warp of eight
    logits[1] = np.where(at // 4096 == 6, np.float32(high), np.float32(low))          # one step
    logits[2] = np.where(at < 4096, np.float32(low), np.float32(high))                # rising
    logits[3] = np.where(at < V - 4096, np.float32(high), np.float32(low))            # falling
    for K in (1, 9, 64):
        check_levels(zlib, logits, scores, K)
    many = np.ascontiguousarray(np.repeat(logits, 90, axis=0))  # stretches of several steps
    check_levels(zlib, many, np.repeat(scores, 90, axis=0), 4)


@pytest.mark.parametrize("K", [1, 8, 64])
@pytest.mark.parametrize("V", [4096, 4097, 20480])
def test_select_nan_ahead_of_equal_logits(zlib, K, V):
    """A NaN counts as -inf among its row's logits, also where all the others are equal."""
    logits = np.zeros((6, 2, V), np.float32)
    logits[0, :, :16] = NAN
    logits[1, :, :200] = NAN
    logits[2, 0, :16] = NAN
    logits[2, 0, V - 3:] = 2.0
    logits[2, 1, 100] = 1.0
    logits[3, 1, ::2] = NAN
    logits[4, 0, :16] = NAN
    logits[4, 0, 16:18] = INF
    logits[4, 1, V - 1] = NAN
    logits[5, :, :8] = NAN
    logits[5, :, 8:] = -3e4
    scores = np.array([[-1, -2]] * 6, np.float32)
    check_select(zlib, logits, scores, None, -1, K)
    check_select(zlib, np.ascontiguousarray(logits[:, :1]), None, None, -1, K)  # one beam fills the selection


def test_select_takes_bool_flags(zlib):
    logits, scores, r = draw(3, 4, 900, 31)
    done = r.random((3, 4)) < 0.4
    want = R.select(logits, scores, done, 2, 6)
    n = zlib.zsaa_op_beam_select_workspace(3, 4, 900, 6)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    s_out, d_out = torch.empty(3, 6, device="cuda"), torch.empty(3, 6, dtype=torch.bool, device="cuda")
    parent, token = (torch.empty(3, 6, dtype=torch.int32, device="cuda") for _ in range(2))
    zlib.zsaa_op_beam_select(torch.from_numpy(logits).cuda(), 900, 3, 4, 900, torch.from_numpy(scores).cuda(),
                             torch.from_numpy(done).cuda(), 2, 6, s_out, parent, token, d_out, ws, n)
    for got, ref in zip((parent, token, d_out), want[1:4]):
        np.testing.assert_array_equal(got.cpu().numpy(), ref)


def test_append_and_reorder_in_a_graph(zlib):
    """Captured calls read the lengths, pages and parents that are there at the replay."""
    p = Pool(zlib, "bf16", 2, 64, 16, 12)
    table = ints([p.row(40, 4, fill=False), p.row(40, 4, fill=False)])
    fresh = ints([p.free.pop() for _ in range(2)])
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    qkv = torch.randn(2, 8 * 64, generator=g, device="cuda").to(torch.bfloat16)
    pos, lens, parent = ints([5, 9]), ints([3, 4]), ints([[0, 1]])
    q, out, out_lens = torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty_like(table), torch.empty_like(lens)
    layers = (zlib.zsaa_pages * 1)(p.pages)

    def step():
        zlib.zsaa_op_paged_append(p.pages, qkv, 512, zlib.ZSAA_BF16, 2, 4, pos, 1e4, None, 2, table, 4, lens, q)
        zlib.zsaa_op_beam_reorder(layers, 1, 2, 2, parent, table, out, 4, lens, out_lens, fresh)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    want = []
    for replay in (False, True):
        p.k.fill_(float("nan"))
        p.v.fill_(float("nan"))
        qkv.copy_(torch.arange(qkv.numel(), device="cuda").view_as(qkv) % 7 - 3)
        pos.copy_(ints([100, 7]))
        lens.copy_(ints([19, 32]))
        parent.copy_(ints([[0, 0]]))
        out.fill_(-9)
        graph.replay() if replay else step()
        torch.cuda.synchronize()
        want.append([torch.nan_to_num(t.float(), nan=-77.0) for t in (p.k, p.v, q, out, out_lens)])
    for a, b in zip(*want):
        assert torch.equal(a, b)
    assert out_lens.tolist() == [19, 19] and out[1, 1] == fresh[1] and out[0, 1] == table[0, 1]
    assert torch.isfinite(p.v[table[0, 1], :, 2]).all() and torch.equal(p.v[table[0, 1], :, 2], p.v[fresh[1], :, 2])


def test_select_in_a_graph(zlib):
    logits, scores, _ = draw(2, 4, 6000, 3)
    x, s = torch.from_numpy(logits).cuda(), torch.from_numpy(scores).cuda()
    n = zlib.zsaa_op_beam_select_workspace(2, 4, 6000, 4)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = [torch.empty(2, 4, device="cuda"), *(torch.empty(2, 4, dtype=torch.int32, device="cuda") for _ in range(2))]

    def call():
        zlib.zsaa_op_beam_select(x, 6000, 2, 4, 6000, s, None, -1, 4, *out, None, ws, n)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    other, other_s, _ = draw(2, 4, 6000, 4)
    x.copy_(torch.from_numpy(other))
    s.copy_(torch.from_numpy(other_s))
    graph.replay()
    torch.cuda.synchronize()
    want = R.select(other, other_s, None, -1, 4)
    np.testing.assert_array_equal(out[1].cpu().numpy(), want[1])
    np.testing.assert_array_equal(out[2].cpu().numpy(), want[2])


# ------------------------------------------------------------------ reorder

@pytest.mark.parametrize("dtype,L,B,W,K,Hkv,hd,page,lens", [
    ("bf16", 1, 1, 1, 1, 1, 64, 16, [0]),
    ("bf16", 2, 1, 1, 4, 2, 64, 16, [21]),          # the first step: one prompt becomes four beams
    ("bf16", 3, 2, 4, 4, 2, 128, 16, [33, 16]),
    ("f32", 2, 3, 3, 5, 1, 32, 32, [1, 31, 100]),
    ("bf16", 64, 1, 2, 2, 1, 64, 64, [63]),
    ("f32", 1, 2, 6, 64, 3, 128, 256, [255, 300]),
])
def test_reorder(zlib, dtype, L, B, W, K, Hkv, hd, page, lens):
    rng = np.random.default_rng(L + B + W + K)
    cols = max(lens) // page + 2
    n_pages = sum(n // page for n in lens) + B * (W + K) + 1
    free = list(rng.permutation(n_pages))
    table = []
    for n in lens:
        whole = [free.pop() for _ in range(n // page)]
        table += [whole + ([free.pop()] if n % page else []) for _ in range(W)]
    table = np.array([t + [-1] * (cols - len(t)) for t in table])
    parent = rng.integers(0, W, (B, K))
    parent[0] = 0  # every slot follows one beam
    fresh = np.array([free.pop() for _ in range(B * K)])
    # the beams of an element may have different lengths within their last page
    each = np.array([n - (n % page) + (int(rng.integers(1, n % page + 1)) if n % page else 0) for n in lens for _ in range(W)])
    k, v = (torch.from_numpy(rng.standard_normal((L, n_pages, Hkv, page, hd)).astype(np.float32)).cuda()
            .to({"bf16": torch.bfloat16, "f32": torch.float32}[dtype]) for _ in range(2))
    want_k, want_v = np64(k), np64(v)
    want, want_lens = R.reorder(want_k, want_v, parent, table, each, fresh, cols)
    out = torch.full((B * K, cols), -9, dtype=torch.int32, device="cuda")
    out_lens = torch.full((B * K,), -9, dtype=torch.int32, device="cuda")
    layers = zlib.make_pages_list(list(k), list(v))
    zlib.zsaa_op_beam_reorder(layers, B, W, K, ints(parent), ints(table), out, cols, ints(each), out_lens, ints(fresh))
    np.testing.assert_array_equal(out.cpu().numpy(), want)
    np.testing.assert_array_equal(out_lens.cpu().numpy(), want_lens)
    np.testing.assert_array_equal(np64(k), want_k)
    np.testing.assert_array_equal(np64(v), want_v)


def test_reorder_a_full_row_has_no_next_page(zlib):
    k = torch.zeros(1, 9, 1, 16, 64, device="cuda")
    layers = zlib.make_pages_list(list(k), list(k.clone()))
    out = torch.full((2, 2), -9, dtype=torch.int32, device="cuda")
    lens = torch.full((2,), -9, dtype=torch.int32, device="cuda")
    zlib.zsaa_op_beam_reorder(layers, 1, 1, 2, ints([[0, 0]]), ints([[5, 3]]), out, 2, ints([32]), lens, ints([7, 8]))
    assert out.tolist() == [[5, 3], [5, 3]] and lens.tolist() == [32, 32]


def test_reorder_reports_bad_parents_lengths_and_pages(zlib):
    k = torch.randn(2, 9, 1, 16, 64, device="cuda")
    v = k.clone()
    before = k.clone()
    layers = zlib.make_pages_list(list(k), list(v))

    def call(parent=(0, 0), table=((5, 3),), lens=(20,), fresh=(7, 8)):
        out, n = ints([[-9, -9]] * 2), ints([-9, -9])
        zlib.zsaa_op_beam_reorder(layers, 1, 1, 2, ints([parent]), ints(table), out, 2, ints(lens), n, ints(fresh))
        with pytest.raises(zlib.ZsaaError) as e:
            zlib.zsaa_device_status()
        assert e.value.status == zlib.ZSAA_ERR_INVALID_ARG
        assert torch.equal(k, before)
        return out.tolist(), n.tolist()

    for p in (-1, 1, 2 ** 31 - 1):
        out, n = call(parent=(0, p))
        assert out == [[5, 3], [-9, -9]] and n == [20, 0]
    for page in (-1, 9, 2 ** 31 - 1):
        call(fresh=(7, page))
        call(table=((5, page),))
    call(lens=(-1,))
    call(lens=(33,))


# ------------------------------------------------------------------ together

class Search:
    """A small decoder (attention and SwiGLU, no norms) whose beams share their prompt."""

    def __init__(self, z, dtype, seed=0):
        self.z, self.dt = z, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        self.code = z.ZSAA_BF16 if dtype == "bf16" else z.ZSAA_F32
        self.d, self.Hq, self.Hkv, self.hd, self.V, self.L, self.F = 256, 4, 2, 64, 4000, 2, 512
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def w(n, k, scale):
            return (scale * torch.randn(n, k, generator=g, device="cuda")).to(self.dt)

        width = (self.Hq + 2 * self.Hkv) * self.hd
        self.embed = w(self.V, self.d, 1.0)
        self.head = w(self.V, self.d, 0.15)
        self.layers = [dict(qkv=w(width, self.d, 0.08), o=w(self.d, self.Hq * self.hd, 0.05), g=w(self.F, self.d, 0.06),
                            u=w(self.F, self.d, 0.06), dn=w(self.d, self.F, 0.04)) for _ in range(self.L)]

    def linear(self, x, W, epi, out_dtype, W2=None, resid=None):
        z, (M, K), N = self.z, x.shape, W.shape[0]
        out = torch.empty(M, N, device="cuda", dtype=out_dtype)
        z.zsaa_op_linear(x, W, W2, resid, out, M, N, K, self.code, epi)
        return out

    def layer(self, l, x, pos, pool, cu, S, table, lens, attention):
        z, lw = self.z, self.layers[l]
        qkv = self.linear(x, lw["qkv"], z.EPI_STORE_F32, torch.float32)
        T = x.shape[0]
        q = torch.empty(T, self.Hq, self.hd, device="cuda", dtype=self.dt)
        z.zsaa_op_paged_append(pool.pages, qkv, qkv.shape[1], z.ZSAA_F32, T, self.Hq, pos, 1e4, cu, S, table,
                               table.shape[1], lens, q)
        a = attention(q).reshape(T, -1)
        x = self.linear(a, lw["o"], z.EPI_RESID, self.dt, resid=x)
        m = self.linear(x, lw["g"], z.EPI_SWIGLU, self.dt, W2=lw["u"])
        return self.linear(m, lw["dn"], z.EPI_RESID, self.dt, resid=x)

    def reference(self, tokens):
        """float64 logits of the last position of one sequence, without a cache."""
        x = np64(self.embed)[np.asarray(tokens)]
        n = len(tokens)
        for lw in self.layers:
            qkv = (x @ np64(lw["qkv"]).T).reshape(n, -1, self.hd)
            qk = R.rope(qkv[:, :self.Hq + self.Hkv], np.arange(n)[:, None], 1e4)
            out = np.zeros((n, self.Hq, self.hd))
            for h in range(self.Hq):
                s = qk[:, h] @ qk[:, self.Hq + h // 2].T / 8.0
                s[np.triu_indices(n, 1)] = -np.inf
                p = np.exp(s - s.max(1, keepdims=True))
                out[:, h] = p / p.sum(1, keepdims=True) @ qkv[:, self.Hq + self.Hkv + h // 2]
            x = x + out.reshape(n, -1) @ np64(lw["o"]).T
            a = x @ np64(lw["g"]).T
            x = x + (a / (1 + np.exp(-a)) * (x @ np64(lw["u"]).T)) @ np64(lw["dn"]).T
        return x[-1] @ np64(self.head).T


@pytest.mark.parametrize("dtype,steps", [("f32", 20), ("bf16", 20)])
def test_a_beam_search_over_shared_prompts(zlib, dtype, steps):
    """Prompts are appended and attended in chunks, then every prompt becomes W beams:
    each step appends, attends over the shared prompt and the beams' pages, selects and
    reorders.  Every chosen continuation's logits are those of its whole sequence without
    a cache, and every choice is the one that the logits at hand ask for."""
    z, m, B, W, page = zlib, Search(zlib, dtype), 2, 3, 16
    rng = np.random.default_rng(1)
    prompts = [list(rng.integers(0, m.V, n)) for n in (37, 16)]
    n_pages = 200
    pools = [Pool(z, dtype, m.Hkv, m.hd, page, n_pages, seed=4) for _ in range(m.L)]
    free = pools[0].free
    plens = [len(p) for p in prompts]
    pcols = max(-(-n // page) for n in plens)
    ptable = ints([[free.pop() for _ in range(-(-n // page))] + [-1] * (pcols - -(-n // page)) for n in plens])
    # the prompts, 8 tokens of each at a time (fewer at the end): a chunk's queries see
    # the entries before it and its own up to theirs
    last = [None] * B
    for b, prompt in enumerate(prompts):
        for at in range(0, len(prompt), 8):
            part = prompt[at:at + 8]
            n = len(part)
            x = m.embed[torch.tensor(part, device="cuda")]
            pos, lens = ints(np.arange(at, at + n)), ints([at + n])
            table = ptable[b:b + 1].contiguous()
            for l in range(m.L):
                x = m.layer(l, x, pos, pools[l], ints([0, n]), 1, table, lens, lambda q: attend_rows(
                    z, pools[l], q.view(1, n, m.Hq, m.hd), table, lens))
        last[b] = x[-1:]
    hidden = torch.cat(last).contiguous()
    cols = steps // page + 2
    beams = 1
    table = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    scores = done = None
    texts = [[list(p)] for p in prompts]
    eos = 3
    tol = (1e-4, 0.0) if dtype == "f32" else (0.0, 2e-2)  # relative to the largest logit; absolute (bf16 storage)
    for step in range(steps):
        logits = m.linear(hidden, m.head, z.EPI_STORE_F32, torch.float32)
        got = np64(logits).reshape(B, beams, m.V)
        for b in range(B):
            for w in range(beams):
                if done is not None and done[b, w]:
                    continue
                ref = m.reference(texts[b][w])
                if dtype == "f32":
                    assert np.abs(got[b, w] - ref).max() <= tol[0] * np.abs(ref).max(), (step, b, w)
                else:
                    rel = np.linalg.norm(got[b, w] - ref) / np.linalg.norm(ref)
                    assert rel <= 2e-2, (step, b, w, rel)
        n = z.zsaa_op_beam_select_workspace(B, beams, m.V, W)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        s_out = torch.empty(B, W, device="cuda")
        parent, token = (torch.empty(B, W, dtype=torch.int32, device="cuda") for _ in range(2))
        d_out = torch.empty(B, W, dtype=torch.uint8, device="cuda")
        z.zsaa_op_beam_select(logits, m.V, B, beams, m.V, scores, done, eos, W, s_out, parent, token, d_out, ws, n)
        want = R.select(logits.cpu().numpy().reshape(B, beams, m.V), None if scores is None else scores.cpu().numpy(),
                        None if done is None else done.cpu().numpy(), eos, W)
        np.testing.assert_array_equal(parent.cpu().numpy(), want[1])
        np.testing.assert_array_equal(token.cpu().numpy(), want[2])
        fresh = [free.pop() for _ in range(B * W)]
        new_table = torch.full((B * W, cols), -1, dtype=torch.int32, device="cuda")
        new_lens = torch.zeros(B * W, dtype=torch.int32, device="cuda")
        layers = (z.zsaa_pages * m.L)(*[p.pages for p in pools])
        z.zsaa_op_beam_reorder(layers, B, beams, W, parent, table, new_table, cols, lens, new_lens, ints(fresh))
        used = set(new_table.flatten().tolist()) | set(ptable.flatten().tolist())
        free[:] = [i for i in range(n_pages) if i not in used]  # pages of beams that ended go back
        texts = [[texts[b][parent[b, j]] + [int(token[b, j])] for j in range(W)] for b in range(B)]
        table, scores, done, beams = new_table, s_out, d_out, W
        lens = new_lens + 1
        x = m.embed[token.view(-1).long()]
        pos = ints([plens[b] + step for b in range(B) for _ in range(W)])
        for l in range(m.L):
            x = m.layer(l, x, pos, pools[l], None, B * W, table, lens, lambda q: attend_rows(
                z, pools[l], q.view(B * W, 1, m.Hq, m.hd), table, lens, ints([0, W, 2 * W]), ptable, ints(plens)))
        hidden = x


def attend_rows(z, pool, q, table, lens, groups=None, ptable=None, plens=None):
    return attend(z, pool, q.contiguous(), table.tolist(), lens.tolist(), None if groups is None else groups.tolist(),
                  None if ptable is None else ptable.tolist(), None if plens is None else plens.tolist())[0]
