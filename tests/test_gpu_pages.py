"""Pages counted by reference on the GPU: resize, fork and compact against plain forms, on
whole pools, tables and counts, so a stray write shows."""

import numpy as np
import pytest
import torch

import paged_ref as R
import pages_ref as P
from helpers import need_gpu, np64
from test_gpu_paged import DTYPES, attend, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(zlib):
    need_gpu()
    yield
    zlib.zsaa_device_status()


def reported(z):
    with pytest.raises(z.ZsaaError) as e:
        z.zsaa_device_status()
    assert e.value.status == z.ZSAA_ERR_INVALID_ARG


def pools(dtype, L, n_pages, Hkv, page, hd, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn(L, n_pages, Hkv, page, hd, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2)]


def out_lens(n):
    return torch.full((n,), -9, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ resize

class Ledger:
    """The device's counts and table beside the plain ones."""

    def __init__(self, z, S, cols, page, n_pages, seed=0):
        self.z, self.S, self.cols, self.page, self.n_pages = z, S, cols, page, n_pages
        self.refs, self.table, self.lens = np.zeros(n_pages, np.int64), np.full((S, cols), -1), np.zeros(S, np.int64)
        r = np.random.default_rng(seed)
        self.refs[r.random(n_pages) < 0.2] = 3  # pages that somebody else holds
        self.d_refs, self.d_table, self.d_lens = ints(self.refs), ints(self.table), ints(self.lens)

    def resize(self, want):
        want = np.asarray(want)
        self.lens, left = P.resize(self.refs, self.page, self.table, self.lens, want)
        n, got = out_lens(1), out_lens(self.S)
        self.z.zsaa_op_paged_resize(self.d_refs, self.n_pages, self.page, self.S, self.d_table, self.cols, self.d_lens, ints(want),
                                    got, n)
        self.d_lens = got
        np.testing.assert_array_equal(self.d_refs.cpu().numpy(), self.refs)
        np.testing.assert_array_equal(self.d_table.cpu().numpy(), self.table)
        np.testing.assert_array_equal(got.cpu().numpy(), self.lens)
        assert n.item() == left


@pytest.mark.parametrize("S,cols,page,n_pages", [
    (1, 1, 16, 1), (1, 300, 16, 310), (3, 5, 256, 40), (7, 200, 32, 700), (64, 9, 64, 257), (65, 3, 16, 5000),
    (1000, 4, 128, 4001), (1025, 2, 16, 1500), (16384, 2, 16, 70001), (5, 129, 16, 300001)])
def test_resize(zlib, S, cols, page, n_pages):
    r = np.random.default_rng(S + cols + n_pages)
    led, cap = Ledger(zlib, S, cols, page, n_pages, seed=S), cols * page
    led.resize(r.integers(0, cap + 1, S))          # (the smaller pools run out of pages)
    led.resize(np.full(S, cap))
    led.resize(r.integers(-3, cap + 1, S))
    led.resize(np.maximum(led.lens + r.integers(-2, 3, S), 0).clip(max=cap))
    led.resize(np.where(r.random(S) < 0.5, led.lens, 0))
    led.resize(led.lens)
    led.resize(np.zeros(S, int))
    assert (led.refs[led.refs != 3] == 0).all()


@pytest.mark.parametrize("n_pages", [600001, 1 << 20, (1 << 20) + 1, (1 << 20) + 300, (1 << 20) + 512, (1 << 20) + 513, 2000000,
                                     (1 << 21) + 1, 5000000, (1 << 30) - 600])
def test_resize_counts_pools_of_which_a_block_is_large(zlib, n_pages):
    """Free pages here and there, the pool's last ones among them: what is left, and what a call gets
    that asks for more than there are."""
    r = np.random.default_rng(n_pages)
    free = np.unique(np.concatenate([r.integers(0, n_pages, 4000), r.integers(n_pages - 200, n_pages, 50), [n_pages - 1]]))
    refs = torch.full((n_pages,), 2, dtype=torch.int32, device="cuda")
    refs[torch.from_numpy(free).cuda()] = 0
    n, got, page, S, cols = len(free), out_lens(3), 16, 3, 3000
    table, lens, left = ints(np.full((S, cols), -1)), ints([0, 0, 0]), out_lens(1)

    def call(want):
        zlib.zsaa_op_paged_resize(refs, n_pages, page, S, table, cols, lens, ints(want), got, left)
        lens.copy_(got)

    call([160, 0, 17])
    assert left.item() == n - 12 and got.tolist() == [160, 0, 17] and (refs == 0).sum().item() == n - 12
    call([2000 * page, 0, 3000 * page])  # (4988 more pages)
    assert left.item() == 0 and got.tolist() == [2000 * page, 0, (n - 2000) * page] and (refs == 0).sum().item() == 0
    taken = np.concatenate([free[:10], free[12:2002], free[10:12], free[2002:]])
    np.testing.assert_array_equal(table.cpu().numpy()[[0] * 2000 + [2] * (n - 2000), [*range(2000), *range(n - 2000)]], taken)
    call([2000 * page, 5 * page, 100 * page])  # what the last one gives up goes to the one before
    assert left.item() == n - 2105 and got.tolist() == [2000 * page, 5 * page, 100 * page]
    call([0, 0, 0])
    assert left.item() == n and (refs == 0).sum().item() == n and refs.sum().item() == 2 * (n_pages - n)


def test_resize_lengths_of_zero_one_and_around_pages(zlib):
    led = Ledger(zlib, 6, 4, 16, 40)
    for want in ([0, 1, 15, 16, 17, 64], [1, 0, 16, 17, 16, 63], [64, 48, 1, 33, 32, 0], [0] * 6):
        led.resize(want)


def test_resize_shared_pages_are_free_when_the_last_reference_goes(zlib):
    led = Ledger(zlib, 8, 3, 16, 64, seed=1)
    led.resize([48] * 4 + [0] * 4)
    led.table[4:], led.lens[4:] = led.table[:4], 40      # four more sequences over the same pages
    np.add.at(led.refs, led.table[4:].ravel(), 1)
    led.d_refs, led.d_table, led.d_lens = ints(led.refs), ints(led.table), ints(led.lens)
    led.resize([0, 16, 48, 1, 40, 0, 33, 17])
    led.resize([16, 0, 0, 0, 0, 0, 0, 0])
    led.resize([48] * 8)


def test_resize_without_a_count_of_free_pages(zlib):
    refs, table, lens, got = ints(np.zeros(9)), ints(np.full((2, 3), -1)), ints([0, 0]), out_lens(2)
    zlib.zsaa_op_paged_resize(refs, 9, 16, 2, table, 3, lens, ints([17, 48]), got)
    assert table.tolist() == [[0, 1, -1], [2, 3, 4]] and got.tolist() == [17, 48]


@pytest.mark.parametrize("page", [-1, 64, 2 ** 31 - 1, -2 ** 31])
def test_resize_reports_pages_out_of_range(zlib, page):
    refs = np.zeros(64, int)
    refs[[5, 6, 7, 8]] = 1
    d_refs, table, got = ints(refs), ints([[5, page], [6, 7], [8, -1]]), out_lens(3)
    zlib.zsaa_op_paged_resize(d_refs, 64, 16, 3, table, 2, ints([32, 32, 16]), ints([16, 0, 32]), got)
    reported(zlib)
    refs[[6, 7]] = 0
    refs[0] = 1  # the third sequence's new page
    assert d_refs.cpu().numpy().tolist() == refs.tolist() and got.tolist() == [16, 0, 32]


def test_resize_reports_pages_that_nobody_holds_and_lengths_beyond_the_row(zlib):
    refs, got = ints([0, 1, 0, 0]), out_lens(2)
    zlib.zsaa_op_paged_resize(refs, 4, 16, 2, ints([[2, 1], [1, 0]]), 2, ints([32, 32]), ints([0, 0]), got)
    reported(zlib)
    assert refs.tolist() == [0, 0, 0, 0] and got.tolist() == [0, 0]
    for lens, want in (([33, 0], [0, 0]), ([0, 0], [33, 0]), ([2 ** 31 - 1, 0], [0, 0]), ([0, 0], [2 ** 31 - 1, 0])):
        refs = ints([1, 1, 0, 0])
        zlib.zsaa_op_paged_resize(refs, 4, 16, 2, ints([[0, 1], [-1, -1]]), 2, ints(lens), ints(want), out_lens(2))
        reported(zlib)
        assert refs.min() >= 0 and refs.max() <= 1


def test_resize_into_a_graph_on_another_stream(zlib):
    """A loop that takes and gives up pages as its lengths say, replayed."""
    S, cols, page, n_pages = 5, 6, 16, 37
    led = Ledger(zlib, S, cols, page, n_pages, seed=3)
    want, out = ints(np.zeros(S)), out_lens(S)

    def call():
        zlib.zsaa_op_paged_resize(led.d_refs, n_pages, page, S, led.d_table, cols, led.d_lens, want, out)
        led.d_lens.copy_(out)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for step in range(6):
            w = np.random.default_rng(step).integers(0, cols * page + 1, S)
            want.copy_(ints(w))
            graph.replay()
            led.lens, _ = P.resize(led.refs, page, led.table, led.lens, w)
            np.testing.assert_array_equal(led.d_refs.cpu().numpy(), led.refs)
            np.testing.assert_array_equal(led.d_table.cpu().numpy(), led.table)
            np.testing.assert_array_equal(led.d_lens.cpu().numpy(), led.lens)


# ------------------------------------------------------------------ fork

def forked(z, dtype, L, Hkv, hd, page, lens, parent, at=None, spare=None, seed=0, pad=1):
    """One fork of parents with lengths `lens`; spare: free pages (None: enough).  Compares
    everything with the plain form and returns the children's lengths."""
    r = np.random.default_rng(seed)
    N, used = len(parent), [P.pages_of(max(n, 0), page) for n in lens]
    cols = max(used + [1]) + pad
    spare = N + 2 if spare is None else spare
    n_pages = sum(used) + spare + 3
    order = r.permutation(n_pages)
    refs, table, i = np.zeros(n_pages, np.int64), np.full((len(lens), cols), -1), 0
    for s, n in enumerate(used):
        table[s, :n] = order[i:i + n]
        i += n
    refs[order[:i]] = 1
    refs[order[i + spare:]] = 2  # held by others
    k, v = pools(dtype, L, n_pages, Hkv, page, hd, seed)
    kk, vv, out = np64(k), np64(v), np.full((N, cols), -9)
    d_refs, d_out, d_lens, left = ints(refs), ints(out), out_lens(N), out_lens(1)
    want, want_left = P.fork(kk, vv, refs, page, table, lens, parent, at, out)
    z.zsaa_op_paged_fork(z.make_pages_list(list(k), list(v)), d_refs, len(lens), ints(table), cols, ints(lens), N, ints(parent),
                         None if at is None else ints(at), d_out, d_lens, left)
    np.testing.assert_array_equal(d_lens.cpu().numpy(), want)
    np.testing.assert_array_equal(d_out.cpu().numpy(), out)
    np.testing.assert_array_equal(d_refs.cpu().numpy(), refs)
    assert left.item() == want_left
    np.testing.assert_array_equal(np64(k), kk)
    np.testing.assert_array_equal(np64(v), vv)
    return want


@pytest.mark.parametrize("dtype,L,Hkv,hd,page,lens,N", [
    ("bf16", 1, 1, 64, 16, [0], 1), ("bf16", 2, 2, 64, 16, [21], 4), ("bf16", 3, 3, 128, 16, [16, 33, 1], 7),
    ("f32", 1, 1, 32, 32, [63, 64, 65], 5), ("f32", 2, 2, 64, 64, [200, 0, 63], 9), ("f32", 1, 5, 128, 256, [255, 511], 3),
    ("bf16", 64, 1, 64, 128, [127], 2), ("bf16", 1, 8, 128, 16, [3000] * 2, 300), ("bf16", 1, 1, 64, 16, [5] * 40, 1500)])
def test_fork(zlib, dtype, L, Hkv, hd, page, lens, N):
    r = np.random.default_rng(N)
    parent = r.integers(0, len(lens), N)
    forked(zlib, dtype, L, Hkv, hd, page, lens, parent)
    at = r.integers(-1, max(lens) + 3, N)
    forked(zlib, dtype, L, Hkv, hd, page, lens, parent, at, pad=0)


def test_fork_no_child_and_every_place_of_a_page(zlib):
    forked(zlib, "bf16", 2, 2, 64, 16, [40], [0] * 34 + [-1] * 3, list(range(34)) + [5, 0, 40])
    forked(zlib, "bf16", 1, 1, 64, 16, [40, -7, 0], [-1, 1, 2, 0])


@pytest.mark.parametrize("spare", [0, 1, 3])
def test_fork_runs_out_of_pages(zlib, spare):
    got = forked(zlib, "bf16", 2, 2, 128, 16, [37, 16, 50, 3], [0, 1, 2, 3, 0, 2], spare=spare)
    assert sorted(got % 16 > 0).count(True) == spare


def test_fork_takes_the_last_pages_of_a_large_pool(zlib):
    """2^20 + 300 pages, the last two free: the third of three children that need one gets none."""
    n_pages, page = (1 << 20) + 300, 16
    k, v = (torch.zeros(1, n_pages, 1, page, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    k[:, :2] = torch.randn(1, 2, 1, page, 64, device="cuda").to(torch.bfloat16)
    refs, out, got, left = torch.ones(n_pages, dtype=torch.int32, device="cuda"), ints(np.full((3, 2), -1)), out_lens(3), out_lens(1)
    refs[n_pages - 2:] = 0
    zlib.zsaa_op_paged_fork(zlib.make_pages_list(list(k), list(v)), refs, 1, ints([[0, 1]]), 2, ints([25]), 3, ints([0, 0, 0]), None,
                            out, got, left)
    assert out.tolist() == [[0, n_pages - 2], [0, n_pages - 1], [0, -1]] and got.tolist() == [25, 25, 16] and left.item() == 0
    assert torch.equal(k[0, -2, 0, :9], k[0, 1, 0, :9]) and torch.equal(k[0, -1, 0, :9], k[0, 1, 0, :9])
    assert refs[0].item() == 4 and (k[0, -2:, 0, 9:] == 0).all()


def test_fork_reports_bad_parents_pages_and_lengths(zlib):
    k, v = pools("bf16", 1, 9, 1, 16, 64, 0)
    before, layers = k.clone(), zlib.make_pages_list(list(k), list(v))

    def call(parent=(0, 0), table=((5, 3),), lens=(20,)):
        refs, out, n = np.zeros(9, int), ints([[-9, -9]] * 2), out_lens(2)
        refs[[3, 5]] = 1
        d_refs = ints(refs)
        zlib.zsaa_op_paged_fork(layers, d_refs, 1, ints(table), 2, ints(lens), 2, ints(parent), None, out, n)
        reported(zlib)
        return d_refs.tolist(), out.tolist(), n.tolist()

    for p in (-2, 1, 2 ** 31 - 1, -2 ** 31):
        refs, out, n = call(parent=(0, p))
        assert refs == [1, 0, 0, 1, 0, 2, 0, 0, 0] and out == [[5, 0], [-9, -9]] and n == [20, 0]
    k.copy_(before)
    for page in (-1, 9, 2 ** 31 - 1):
        call(table=((5, page),))
        refs, _, _ = call(table=((page, 3),), lens=(16,))
        assert refs == [0, 0, 0, 1, 0, 1, 0, 0, 0]
        assert torch.equal(k, before)
    call(lens=(33,))


# ------------------------------------------------------------------ compact

def compacted(z, dtype, L, Hkv, hd, page, lens, keep, start=None, moved=False, counted=False, seed=0):
    r = np.random.default_rng(seed)
    used = [P.pages_of(n, page) for n in lens]
    ends = [(0 if start is None else start[s]) + len(x) for s, x in enumerate(keep)]
    cols, out_cols = max(used + [1]), max([P.pages_of(n, page) for n in ends] + [1])
    n_pages = sum(used) + (sum(P.pages_of(n, page) for n in ends) if moved else 0) + 2
    free = list(r.permutation(n_pages))
    row = lambda n, cols: [free.pop() for _ in range(P.pages_of(n, page))] + [-1] * (cols - P.pages_of(n, page))
    table = np.array([row(n, cols) for n in lens])
    out = np.array([row(n, out_cols) for n in ends]) if moved else table
    width = max(len(x) for x in keep) + 1
    listed = np.full((len(lens), width), -5)
    for s, x in enumerate(keep):
        listed[s, :len(x)] = x
    n_keep = [len(x) for x in keep]
    refs = np.zeros(n_pages, int)
    refs[out[out >= 0]] = 1
    k, v = pools(dtype, L, n_pages, Hkv, page, hd, seed)
    kk, vv = np64(k), np64(v)
    want = P.compact(kk, vv, page, table, start, listed, n_keep, out)
    got, d_table = out_lens(len(lens)), ints(table)
    d_out = ints(out) if moved else d_table
    z.zsaa_op_paged_compact(z.make_pages_list(list(k), list(v)), ints(refs) if counted else None, len(lens), d_table, cols,
                            ints(lens), None if start is None else ints(start), ints(listed), width, ints(n_keep), d_out,
                            out.shape[1], got)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    np.testing.assert_array_equal(np64(k), kk)
    np.testing.assert_array_equal(np64(v), vv)
    np.testing.assert_array_equal(d_table.cpu().numpy(), table)


def some_of(r, lens, share, start=None):
    keep = []
    for s, n in enumerate(lens):
        a = 0 if start is None else start[s]
        keep.append(np.sort(r.permutation(n - a)[:int(round(share * (n - a)))]) + a)
    return keep


@pytest.mark.parametrize("moved", [False, True])
@pytest.mark.parametrize("dtype,L,Hkv,hd,page,lens", [
    ("bf16", 1, 1, 64, 16, [1]), ("bf16", 2, 3, 64, 16, [33, 0, 16, 17]), ("bf16", 1, 8, 128, 64, [900, 63]),
    ("f32", 2, 4, 32, 16, [77, 200, 31]), ("f32", 1, 2, 64, 32, [500]), ("f32", 3, 1, 128, 128, [300, 128]),
    ("bf16", 64, 2, 128, 256, [700]), ("bf16", 1, 1, 64, 16, [9001, 40]), ("bf16", 2, 2, 128, 16, list(range(0, 90)))])
def test_compact(zlib, dtype, L, Hkv, hd, page, lens, moved):
    r = np.random.default_rng(len(lens) + max(lens))
    for i, share in enumerate((0.5, 0.1, 1.0, 0.0, 0.93)):
        compacted(zlib, dtype, L, Hkv, hd, page, lens, some_of(r, lens, share), moved=moved, counted=i % 2 == 1, seed=i)
    start = [int(r.integers(0, n + 1)) for n in lens]
    for share in (0.4, 1.0):
        compacted(zlib, dtype, L, Hkv, hd, page, lens, some_of(r, lens, share, start), start, moved=moved, counted=True)


@pytest.mark.parametrize("moved", [False, True])
def test_compact_runs_shifts_and_ends(zlib, moved):
    """What a window with its first entries kept leaves; one entry dropped at either end; the
    last entries alone."""
    n = 3000
    for keep in ([*range(4), *range(2000, n)], range(1, n), range(n - 1), [n - 1], [0], range(n - 17, n), range(0, n, 2),
                 [i for i in range(n) if i % 16], [*range(512), *range(513, n)]):
        compacted(zlib, "bf16", 1, 2, 64, 16, [n], [list(keep)], moved=moved)
        compacted(zlib, "f32", 1, 1, 128, 64, [n], [list(keep)], moved=moved)


@pytest.mark.parametrize("counted", [False, True])
@pytest.mark.parametrize("same", ["all", "first", "last", "one"])
@pytest.mark.parametrize("dtype,L,Hkv,hd,page,lens", [
    ("bf16", 1, 1, 64, 16, [9001]), ("bf16", 2, 3, 128, 32, [333, 40, 0, 700]), ("f32", 1, 2, 32, 16, [5, 900]),
    ("f32", 1, 4, 128, 64, [3000])])
def test_compact_by_another_array_that_names_the_same_pages(zlib, dtype, L, Hkv, hd, page, lens, same, counted):
    """table_out is no part of table, but some or all of its columns are the same: in place as far as
    those go.  (The first shape is planned for several clusters to its list, and one does it.)"""
    z, r = zlib, np.random.default_rng(len(same) + len(lens))
    used = [P.pages_of(n, page) for n in lens]
    cols = max(used)
    out_cols = cols + 2
    n_pages = 2 * sum(used) + 1
    free = list(r.permutation(n_pages))
    table, out = np.full((len(lens), cols), -1), np.full((len(lens), out_cols), -1)
    for s, n in enumerate(used):
        table[s, :n] = [free.pop() for _ in range(n)]
        cut = r.integers(0, n + 1)
        for c in range(n):
            keeps = dict(all=True, first=c < cut, last=c >= cut, one=c == cut)[same]
            out[s, c] = table[s, c] if keeps else free.pop()
    keep = some_of(r, lens, 0.6)
    width = max(len(x) for x in keep)
    listed = np.zeros((len(lens), width), int)
    for s, x in enumerate(keep):
        listed[s, :len(x)] = x
    refs = np.zeros(n_pages, int)
    refs[out[out >= 0]] = 1
    k, v = pools(dtype, L, n_pages, Hkv, page, hd, 4)
    kk, vv, got = np64(k), np64(v), out_lens(len(lens))
    want = P.compact(kk, vv, page, table, None, listed, [len(x) for x in keep], out)
    z.zsaa_op_paged_compact(z.make_pages_list(list(k), list(v)), ints(refs) if counted else None, len(lens), ints(table), cols,
                            ints(lens), None, ints(listed), width, ints([len(x) for x in keep]), ints(out), out_cols, got)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    np.testing.assert_array_equal(np64(k), kk)
    np.testing.assert_array_equal(np64(v), vv)


@pytest.mark.parametrize("out_cols", [2, 5])
def test_compact_of_one_sequence_in_place_by_a_row_of_another_width(zlib, out_cols):
    """One row that starts where the table does is the same row, as far as it goes."""
    k, v = pools("bf16", 1, 6, 1, 16, 64, 0)
    kk, vv, keep = np64(k), np64(v), np.array([[1, 5, *range(20, 48)]])
    table, got = ints([[3, 1, 4, -1, -1]]), out_lens(1)
    P.compact(kk, vv, 16, np.array([[3, 1, 4]]), None, keep, [30], np.array([[3, 1]]))
    zlib.zsaa_op_paged_compact(zlib.make_pages_list(list(k), list(v)), None, 1, table, 3, ints([48]), None, ints(keep), 30, ints([30]),
                               table, out_cols, got)
    assert got.tolist() == [30]
    np.testing.assert_array_equal(np64(k), kk)
    np.testing.assert_array_equal(np64(v), vv)


@pytest.mark.parametrize("n", [40, 5000])
def test_compact_moves_a_pool_that_several_layers_name_once(zlib, n):
    """Layers that share a cache, and one whose keys are its values."""
    z, page = zlib, 16
    used = P.pages_of(n, page)
    k, v = pools("bf16", 3, used, 2, page, 64, n)
    kk, vv, table = np64(k), np64(v), np.arange(used)[None]
    keep = np.sort(np.random.default_rng(n).permutation(n)[:n * 2 // 3])
    P.compact(kk, vv, page, table, None, keep[None], [len(keep)], table)
    layers = z.make_pages_list([k[0], k[1], k[0], k[2], v[0], k[1]], [v[0], v[1], v[0], k[2], v[2], v[0]])
    d_table, got = ints(table), out_lens(1)
    z.zsaa_op_paged_compact(layers, None, 1, d_table, used, ints([n]), None, ints([keep]), len(keep), ints([len(keep)]), d_table, used,
                            got)
    np.testing.assert_array_equal(np64(k), kk)
    np.testing.assert_array_equal(np64(v), vv)


def test_compact_leaves_shared_pages_alone_where_it_moves_nothing(zlib):
    """Two sequences over one whole page, each with a page of its own: the kept entries of the
    shared page stay where they are, and with counts that is allowed."""
    k, v = pools("bf16", 2, 5, 2, 16, 64, 3)
    kk, vv, table = np64(k), np64(v), np.array([[0, 1], [0, 2]])
    keep = np.array([[*range(16), 18, 19, 25], [*range(16), 17, 30, 31]])
    want = P.compact(kk, vv, 16, table, None, keep, [19, 19], table)
    got, layers = out_lens(2), zlib.make_pages_list(list(k), list(v))
    d_table, refs = ints(table), ints([2, 1, 1, 0, 0])
    zlib.zsaa_op_paged_compact(layers, refs, 2, d_table, 2, ints([32, 32]), None, ints(keep), 19, ints([19, 19]), d_table, 2, got)
    assert got.tolist() == want.tolist()
    np.testing.assert_array_equal(np64(k), kk)
    np.testing.assert_array_equal(np64(v), vv)
    before = k.clone()
    keep = ints([[1, 2], [1, 2]])  # this would write the shared page
    zlib.zsaa_op_paged_compact(layers, refs, 2, d_table, 2, ints([32, 32]), None, keep, 2, ints([2, 2]), d_table, 2, got)
    reported(zlib)
    assert torch.equal(k, before)


@pytest.mark.parametrize("bad", [dict(keep=[0, 32, 20]), dict(keep=[3, 3, 4]), dict(keep=[5, 4, 6]), dict(keep=[-1, 4, 6]),
                                 dict(lens=[33]), dict(table=[[4, 9]]), dict(table=[[-1, 5]]), dict(n_keep=[4]), dict(start=[33]),
                                 dict(start=[30]), dict(out=[[9, 5]]), dict(out=[[2 ** 31 - 1, 5]])])
def test_compact_reports_what_is_out_of_range(zlib, bad):
    f = dict(keep=[1, 17, 30], lens=[32], table=[[4, 5]], n_keep=[3], start=None, out=[[6, 7]])
    f.update(bad)
    k, v = pools("bf16", 1, 9, 1, 16, 64, 0)
    before, got = k.clone(), out_lens(1)
    zlib.zsaa_op_paged_compact(zlib.make_pages_list(list(k), list(v)), None, 1, ints(f["table"]), 2, ints(f["lens"]),
                               None if f["start"] is None else ints(f["start"]), ints([f["keep"]]), 3, ints(f["n_keep"]),
                               ints(f["out"]), 2, got)
    reported(zlib)
    assert torch.equal(k[:, [0, 1, 2, 3, 4, 5, 8]], before[:, [0, 1, 2, 3, 4, 5, 8]])  # nothing but the pages of the result
    assert 0 <= got.item() <= 32


def test_compact_into_rows_too_short(zlib):
    """A result that its table row does not hold is cut, and reported."""
    k, v = pools("bf16", 1, 6, 1, 16, 64, 0)
    before, got = k.clone(), out_lens(1)
    zlib.zsaa_op_paged_compact(zlib.make_pages_list(list(k), list(v)), None, 1, ints([[0, 1]]), 2, ints([32]), None,
                               ints([list(range(2, 22))]), 20, ints([20]), ints([[5]]), 1, got)
    reported(zlib)
    assert got.tolist() == [16] and torch.equal(k[0, 5, 0, :14], before[0, 0, 0, 2:]) and torch.equal(k[0, :5], before[0, :5])


@pytest.mark.parametrize("n_keep", [0, 3])
def test_compact_from_beyond_the_row_it_writes(zlib, n_keep):
    """Entries below `start` that the other row has no place for: its length is what it holds, and
    that is reported."""
    k, v = pools("bf16", 1, 6, 1, 16, 64, 0)
    before, got, layers = k.clone(), out_lens(2), zlib.make_pages_list(list(k), list(v))

    def call(start):
        zlib.zsaa_op_paged_compact(layers, None, 2, ints([[0, 1], [2, 3]]), 2, ints([32, 32]), ints([0, start]),
                                   ints([[4, 5, 6], [28, 29, 31]]), 3, ints([0, n_keep]), ints([[4], [5]]), 1, got)

    call(17)
    reported(zlib)
    assert got.tolist() == [0, 16] and torch.equal(k, before)
    if n_keep == 0:
        call(16)  # (and nothing to report: 16 entries below the start fill the row)
        assert got.tolist() == [0, 16] and torch.equal(k, before)


def test_pages_far_into_a_large_pool(zlib):
    """Element offsets past 2^31: the last pages of pools of 5 GB."""
    z, n_pages, page = zlib, 40000, 64
    k, v = (torch.empty(1, n_pages, 8, page, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    last = list(range(n_pages - 4, n_pages))
    for x in (k, v):
        x[:, last] = torch.randn(1, 4, 8, page, 128, device="cuda").to(torch.bfloat16)
    kk, vv = np64(k[:, last]), np64(v[:, last])
    layers = z.make_pages_list(list(k), list(v))
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    refs[n_pages - 2:] = 0
    table, got, out = ints([[n_pages - 4, n_pages - 3]]), out_lens(1), ints([[-1, -1]])
    z.zsaa_op_paged_fork(layers, refs, 1, table, 2, ints([100]), 1, ints([0]), None, out, got)
    assert out.tolist() == [[n_pages - 4, n_pages - 2]] and got.tolist() == [100]
    rel, r_refs, r_out = np.array([[0, 1]]), np.array([1, 1, 0, 0]), np.array([[-1, -1]])
    P.fork(kk, vv, r_refs, page, rel, [100], [0], None, r_out)
    keep = np.sort(np.random.default_rng(0).permutation(100)[:70])
    z.zsaa_op_paged_compact(layers, None, 1, table, 2, ints([100]), None, ints([keep]), 70, ints([70]), table, 2, got)
    P.compact(kk, vv, page, rel, None, keep[None], [70], rel)
    np.testing.assert_array_equal(np64(k[:, last]), kk)
    np.testing.assert_array_equal(np64(v[:, last]), vv)


def test_fork_and_compact_into_a_graph_on_another_stream(zlib):
    """Samples of a prompt that lose half of their entries, released and made again by a replayed
    graph, as their parents' lengths and the entries chosen change."""
    z, page, S, N, cols, n_pages = zlib, 16, 2, 4, 5, 40
    k, v = pools("bf16", 2, n_pages, 2, page, 64, 9)
    layers = z.make_pages_list(list(k), list(v))
    refs, table, lens = ints(np.zeros(n_pages)), ints(np.full((S, cols), -1)), out_lens(S)
    z.zsaa_op_paged_resize(refs, n_pages, page, S, table, cols, ints([0] * S), ints([cols * page] * S), lens)
    kids, kid_lens, half, zero, parent = ints(np.full((N, cols), -1)), ints([0] * N), ints([0] * N), ints([0] * N), ints([0, 1, 1, 0])
    at, keep, n_keep, own, left = ints([1] * N), ints(np.zeros((N, 40))), ints([0] * N), ints(np.full((N, cols), -1)), out_lens(N)

    def call():
        z.zsaa_op_paged_resize(refs, n_pages, page, N, own, cols, half, zero, left)
        z.zsaa_op_paged_fork(layers, refs, S, table, cols, lens, N, parent, at, kids, kid_lens)
        z.zsaa_op_paged_resize(refs, n_pages, page, N, own, cols, zero, n_keep, half)
        z.zsaa_op_paged_compact(layers, refs, N, kids, cols, kid_lens, None, keep, 40, n_keep, own, cols, half)
        z.zsaa_op_paged_resize(refs, n_pages, page, N, kids, cols, kid_lens, zero, left)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for step in range(4):
            r = np.random.default_rng(step)
            sizes = r.integers(2, 70, N)
            chosen = [np.sort(r.permutation(n)[:n // 2]) for n in sizes]
            rows = np.zeros((N, 40), int)
            for i, c in enumerate(chosen):
                rows[i, :len(c)] = c
            at.copy_(ints(sizes)), keep.copy_(ints(rows)), n_keep.copy_(ints([len(c) for c in chosen]))
            kk, vv = np64(k), np64(v)
            graph.replay()
            torch.cuda.synchronize()
            assert refs.sum().item() == S * cols + sum(-(-len(c) // page) for c in chosen) and half.tolist() == [len(c) for c in chosen]
            for i, c in enumerate(chosen):
                for pool, was in ((np64(k), kk), (np64(v), vv)):
                    for l in range(2):
                        have = R.entries(pool[l], own[i].tolist(), len(c))
                        np.testing.assert_array_equal(have, R.entries(was[l], table[parent[i]].tolist(), sizes[i])[:, c])


def test_a_cache_is_pruned_and_attended(zlib):
    """Scores choose half of each sequence's entries, the cache is compacted and its pages are
    given up; attention then sees exactly the chosen entries.  Forks of a sequence prune on
    pages of their own."""
    z, Hq, Hkv, hd, page, S, n = zlib, 8, 2, 64, 16, 3, 100
    k, v = pools("bf16", 1, 60, Hkv, page, hd, 5)
    layers = z.make_pages_list(list(k), list(v))
    cols, refs = 8, torch.zeros(60, dtype=torch.int32, device="cuda")
    table, zero, lens = torch.full((S, cols), -1, dtype=torch.int32, device="cuda"), ints([0] * S), out_lens(S)
    z.zsaa_op_paged_resize(refs, 60, page, S, table, cols, zero, ints([n] * S), lens)
    # two more sequences continue the first from its middle
    kid_table, kid_lens = torch.full((2, cols), -1, dtype=torch.int32, device="cuda"), out_lens(2)
    z.zsaa_op_paged_fork(layers, refs, S, table, cols, lens, 2, ints([0, 0]), ints([50, 41]), kid_table, kid_lens)
    assert kid_lens.tolist() == [50, 41] and (refs == 3).sum().item() == 2 and (refs == 2).sum().item() == 1
    hidden = torch.randn(2, 50, 64, device="cuda").to(torch.bfloat16)
    idx = ints(np.zeros((2, 20)))
    z.zsaa_score_select(hidden[:, :41].contiguous(), 2, 41, 64, 20, idx)
    # the forks' results go to pages of their own, then they give up the shared ones
    own_table, own_lens = torch.full((2, cols), -1, dtype=torch.int32, device="cuda"), out_lens(2)
    z.zsaa_op_paged_resize(refs, 60, page, 2, own_table, cols, ints([0, 0]), ints([20, 20]), own_lens)
    got = out_lens(2)
    kk, vv = np64(k)[0], np64(v)[0]
    z.zsaa_op_paged_compact(layers, refs, 2, kid_table, cols, kid_lens, None, idx, 20, ints([20, 20]), own_table, cols, got)
    z.zsaa_op_paged_resize(refs, 60, page, 2, kid_table, cols, kid_lens, ints([0, 0]), out_lens(2))
    assert got.tolist() == [20, 20] and refs.max().item() == 1 and refs.sum().item() == 3 * 7 + 2 * 2
    q = torch.randn(2, 1, Hq, hd, device="cuda").to(torch.bfloat16)

    class Pages:
        pages = layers[0]

    out, _ = attend(z, Pages, q, own_table.tolist(), [20, 20])
    for s in range(2):
        rows = [R.entries(x, kid_table[s].tolist(), 41)[:, idx[s].tolist()] for x in (kk, vv)]
        pool = [np.concatenate([x, np.zeros((Hkv, 12, hd))], 1).reshape(Hkv, 2, page, hd).transpose(1, 0, 2, 3) for x in rows]
        w = {}
        ref, _ = R.attention(pool[0], pool[1], np64(q)[s:s + 1], [[0, 1]], [20], weighted=w)
        tol, _ = R.attention_tol(ref, w, 21, hd, True)
        assert np.all(np.abs(np64(out)[s:s + 1] - ref) <= tol)
