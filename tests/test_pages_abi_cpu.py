"""Argument checks of the calls over counted pages and of draft verification: refused on
the host, before any device work (the addresses below are never dereferenced)."""

import ctypes as C

import numpy as np
import pytest

import pages_ref as P
from test_paged_abi_cpu import A, BAD_PAGES, FAR, UNSUPPORTED_PAGES, pages, refused

B, D, E = FAR + (1 << 36), FAR + (2 << 36), FAR + (3 << 36)


def resize(z, **kw):
    f = dict(refs=A, n_pages=64, page_size=16, S=4, table=B, cols=5, lens=D, want=E, lens_out=FAR, n_free=None)
    f.update(kw)
    z.zsaa_op_paged_resize(*f.values(), stream=0)


def fork(z, layers=None, **kw):
    f = dict(refs=A, S=4, table=B, cols=5, lens=D, N=6, parent=E, at=E + 4096, table_out=FAR, lens_out=FAR + 4096, n_free=None)
    f.update(kw)
    layers = layers or [pages(z), pages(z)]
    z.zsaa_op_paged_fork((z.zsaa_pages * len(layers))(*layers), *f.values(), stream=0)


def compact(z, layers=None, **kw):
    f = dict(refs=A, S=4, table=B, cols=5, lens=D, start=None, keep=E, keep_cols=30, n_keep=D + 4096, table_out=B, out_cols=5,
             lens_out=FAR)
    f.update(kw)
    layers = layers or [pages(z), pages(z)]
    z.zsaa_op_paged_compact((z.zsaa_pages * len(layers))(*layers), *f.values(), stream=0)


def verify(z, **kw):
    f = dict(target=A, ld=1000, draft=B, draft_ld=1000, dtype=z.ZSAA_F32, S=4, n=3, V=1000, drafts=D, temperature=None,
             uniform=E, accepted=FAR, tokens=FAR + 4096, logp=None, lens=None, lens_out=None, ws=A, ws_bytes=1 << 40)
    f.update(kw)
    z.zsaa_op_draft_verify(*f.values(), stream=0)


@pytest.mark.parametrize("kw", [
    dict(refs=None), dict(table=None), dict(lens=None), dict(want=None), dict(lens_out=None), dict(n_pages=0),
    dict(n_pages=(1 << 30) + 1), dict(S=0), dict(cols=0), dict(cols=1 << 28), dict(S=16384, cols=1 << 18), dict(refs=A + 2),
    dict(table=B + 1), dict(lens=D + 2), dict(want=E + 2), dict(lens_out=FAR + 2), dict(n_free=A + 1), dict(lens_out=D + 4),
    dict(lens_out=E)])
def test_resize_refusals(zlib, kw):
    refused(zlib, lambda: resize(zlib, **kw))


@pytest.mark.parametrize("kw", [dict(page_size=0), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(S=16385)])
def test_resize_refuses_what_it_does_not_support(zlib, kw):
    refused(zlib, lambda: resize(zlib, **kw), zlib.ZSAA_ERR_UNSUPPORTED)


@pytest.mark.parametrize("kw", BAD_PAGES + UNSUPPORTED_PAGES)
def test_pools_are_checked(zlib, kw):
    st = zlib.ZSAA_ERR_UNSUPPORTED if kw in UNSUPPORTED_PAGES else None
    refused(zlib, lambda: fork(zlib, [pages(zlib), pages(zlib, **kw)]), st)
    refused(zlib, lambda: compact(zlib, [pages(zlib, **kw), pages(zlib)]), st)


@pytest.mark.parametrize("kw", [
    dict(refs=None), dict(table=None), dict(lens=None), dict(parent=None), dict(table_out=None), dict(lens_out=None), dict(S=0),
    dict(N=0), dict(cols=0), dict(cols=1 << 28), dict(S=1 << 30), dict(refs=A + 2), dict(table=B + 2), dict(lens=D + 1),
    dict(parent=E + 2), dict(at=E + 1), dict(table_out=FAR + 2), dict(lens_out=FAR + 1), dict(n_free=A + 2),
    dict(table_out=B + 40), dict(lens_out=D), dict(lens_out=E + 8), dict(lens_out=E + 4096)])
def test_fork_refusals(zlib, kw):
    refused(zlib, lambda: fork(zlib, **kw))


def test_fork_refuses_more_children_than_it_takes(zlib):
    refused(zlib, lambda: fork(zlib, N=16385), zlib.ZSAA_ERR_UNSUPPORTED)


@pytest.mark.parametrize("kw", [
    dict(table=None), dict(lens=None), dict(keep=None), dict(n_keep=None), dict(table_out=None), dict(lens_out=None), dict(S=0),
    dict(keep_cols=0), dict(cols=0), dict(out_cols=0), dict(cols=1 << 28), dict(out_cols=1 << 28), dict(refs=A + 2),
    dict(table=B + 2), dict(lens=D + 1), dict(start=D + 2), dict(keep=E + 2), dict(n_keep=D + 4097), dict(table_out=FAR + 1),
    dict(lens_out=FAR + 2), dict(lens_out=D + 8), dict(lens_out=D + 4096), dict(start=D + 8192, lens_out=D + 8196)])
def test_compact_refusals(zlib, kw):
    refused(zlib, lambda: compact(zlib, **kw))


OVER = "overlaps another array"


@pytest.mark.parametrize("kw", [
    dict(n_free=D), dict(n_free=D + 12), dict(n_free=E + 4), dict(n_free=FAR), dict(n_free=A + 4 * 63), dict(n_free=B + 4 * 19),
    dict(lens_out=A + 4 * 63), dict(lens_out=B - 12), dict(table=A + 4 * 63), dict(lens=A), dict(want=B + 76), dict(lens=D, want=A - 12)])
def test_resize_refuses_arrays_over_what_it_writes(zlib, kw):
    with pytest.raises(zlib.ZsaaError, match=OVER):
        resize(zlib, **kw)


@pytest.mark.parametrize("kw", [
    dict(n_free=D + 12), dict(n_free=E + 20), dict(n_free=E + 4096), dict(n_free=B + 76), dict(n_free=FAR + 116), dict(n_free=FAR + 4096),
    dict(n_free=A), dict(table_out=D - 116), dict(table_out=E), dict(table_out=E + 4100), dict(table_out=A + 252), dict(lens_out=B + 76),
    dict(lens_out=A), dict(lens_out=FAR + 100), dict(lens=A), dict(parent=A + 240), dict(table=A)])
def test_fork_refuses_arrays_over_what_it_writes(zlib, kw):
    with pytest.raises(zlib.ZsaaError, match=OVER):
        fork(zlib, **kw)


@pytest.mark.parametrize("kw", [
    dict(lens_out=B + 76), dict(lens_out=E + 4 * 119), dict(lens_out=E - 12), dict(table_out=FAR - 76), dict(refs=FAR - 252)])
def test_compact_refuses_lengths_over_another_array(zlib, kw):
    with pytest.raises(zlib.ZsaaError, match=OVER):
        compact(zlib, **kw)


@pytest.mark.parametrize("kw", [
    dict(out_cols=4), dict(out_cols=6), dict(out_cols=6, S=2), dict(table_out=B + 4), dict(table_out=B + 76), dict(table_out=B - 76),
    dict(table_out=B + 20), dict(table_out=B + 4, S=1), dict(table_out=B + 4, S=1, out_cols=4)])
def test_compact_refuses_tables_that_overlap_otherwise_than_in_place(zlib, kw):
    with pytest.raises(zlib.ZsaaError, match="table_out overlaps table"):
        compact(zlib, **kw)


@pytest.mark.parametrize("call,kw", [
    (compact, dict()), (compact, dict(S=1, out_cols=3)), (compact, dict(S=1, out_cols=9)), (compact, dict(table_out=B + 80)),
    (compact, dict(table_out=B - 80)), (resize, dict(n_free=D + 16)), (resize, dict(n_free=A + 256)), (resize, dict(want=D)), (resize, dict(lens_out=B + 80)),
    (fork, dict(n_free=FAR + 120)), (fork, dict(table_out=B + 80, lens_out=D + 16)), (fork, dict(at=E)), (fork, dict(n_free=A - 4)),
    (compact, dict(lens_out=B + 80)), (compact, dict(lens_out=D + 16)), (compact, dict(refs=FAR + 16))])
def test_arrays_side_by_side_are_taken(zlib, call, kw):
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a device, and the addresses are none of its")
    refused(zlib, lambda: call(zlib, **kw), zlib.ZSAA_ERR_CUDA)


def test_unlike_layers_and_their_number(zlib):
    for kw in (dict(n_pages=65), dict(page_size=32), dict(n_kv_heads=1), dict(head_dim=128)):
        refused(zlib, lambda: fork(zlib, [pages(zlib), pages(zlib, **kw)]))
        refused(zlib, lambda: compact(zlib, [pages(zlib), pages(zlib, **kw)]))
    refused(zlib, lambda: fork(zlib, [pages(zlib)] * 65))
    refused(zlib, lambda: compact(zlib, [pages(zlib)] * 65))
    for call in (fork, compact):
        refused(zlib, lambda: call(zlib, [pages(zlib, n_kv_heads=16384, n_pages=1)]))
    L, one = zlib.lib(), pages(zlib)
    for layers, n in ((None, 1), (C.addressof(one), 0)):
        assert L.zsaa_op_paged_fork(layers, n, A, 1, B, 1, D, 1, E, None, FAR, FAR + 64, None, None) == zlib.ZSAA_ERR_INVALID_ARG
        assert L.zsaa_op_paged_compact(layers, n, None, 1, B, 1, D, None, E, 1, D + 64, B, 1, FAR, None) == zlib.ZSAA_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(target=None), dict(drafts=None), dict(uniform=None), dict(accepted=None), dict(tokens=None), dict(ws=None), dict(S=0),
    dict(V=0), dict(V=(1 << 26) + 1, ld=1 << 27, draft_ld=1 << 27), dict(dtype=5), dict(ld=999), dict(draft_ld=999),
    dict(ld=(1 << 40) + 1), dict(target=A + 2), dict(draft=B + 1), dict(drafts=D + 2), dict(temperature=E + 2),
    dict(uniform=E + 1), dict(accepted=FAR + 2), dict(tokens=FAR + 4098), dict(logp=E + 2), dict(ws=A + 8), dict(ws_bytes=64),
    dict(lens=A), dict(lens_out=A), dict(lens=D + 4096, lens_out=D + 4100), dict(tokens=D + 12), dict(S=1 << 27),
    dict(lens=A + 2, lens_out=A + 2)])
def test_verify_refusals(zlib, kw):
    refused(zlib, lambda: verify(zlib, **kw))


@pytest.mark.parametrize("kw", [
    dict(logp=E), dict(logp=E + 60), dict(accepted=E + 12), dict(tokens=E - 4), dict(temperature=B, logp=B + 12), dict(accepted=D),
    dict(accepted=FAR + 4096 - 12), dict(logp=FAR + 4096), dict(lens=B, lens_out=FAR + 12), dict(lens=B, lens_out=E),
    dict(accepted=B, lens=B, lens_out=B + 4096), dict(lens=B, lens_out=B, temperature=B + 12)])
def test_verify_refuses_outputs_over_anything_else(zlib, kw):
    refused(zlib, lambda: verify(zlib, **kw))


W = FAR + (5 << 36)  # a workspace apart from everything else
TARGET, DRAFT = (15 * 1024 + 1000) * 4, (11 * 1100 + 1000) * 4  # bytes of rows 1024 and 1100 apart


@pytest.mark.parametrize("kw,what", [
    (dict(accepted=A), "logits"), (dict(accepted=A - 12), "logits"), (dict(accepted=A + TARGET - 4), "logits"),
    (dict(accepted=A + 4 * 1021), "logits"), (dict(accepted=A + 4 * (7 * 1024 + 999)), "logits"), (dict(tokens=A + 4 * 1010), "logits"),
    (dict(logp=B + 4), "logits"), (dict(logp=B + DRAFT - 4), "logits"), (dict(logp=B + 4 * 1090), "logits"),
    (dict(lens=D + 4096, lens_out=B + 4 * 2200), "logits"), (dict(ws=A), "logits"), (dict(ws=B + 4 * 2196), "logits"),
    (dict(ws=B - 64), "logits"), (dict(lens=A, lens_out=A), "logits"), (dict(ws=D), "array"), (dict(ws=E), "array"), (dict(ws=FAR), "array"),
    (dict(ws=FAR + 4096 + 48), "array"), (dict(logp=W + 16), "array"), (dict(temperature=W + 64), "array"),
    (dict(lens=W, lens_out=FAR + 8192), "array"), (dict(lens=D + 4096, lens_out=W), "array")])
def test_verify_refuses_outputs_and_a_workspace_over_logits_or_one_another(zlib, kw, what):
    with pytest.raises(zlib.ZsaaError, match="overlaps " + ("the logits" if what == "logits" else "another array")):
        verify(zlib, **{**dict(ld=1024, draft_ld=1100, ws=W), **kw})


@pytest.mark.parametrize("kw", [
    dict(), dict(accepted=A + 4 * 1000), dict(accepted=A + 4 * 1020), dict(accepted=A + TARGET), dict(accepted=A - 16),
    dict(logp=B + 4 * 1000), dict(logp=B + DRAFT), dict(logp=B + 4 * 1084), dict(lens=A, lens_out=FAR + 8192), dict(draft=A),
    dict(ws=A + TARGET), dict(lens=FAR + 8192, lens_out=FAR + 8192), dict(n=0, drafts=A, draft=FAR)])
def test_verify_takes_outputs_beside_and_between_rows_of_logits(zlib, kw):
    """Nothing refuses them before a device is looked for."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a device, and the addresses are none of its")
    refused(zlib, lambda: verify(zlib, **{**dict(ld=1024, draft_ld=1100, ws=W), **kw}), zlib.ZSAA_ERR_CUDA)


@pytest.mark.parametrize("n", [-1, 16])
def test_verify_refuses_more_drafts_than_it_takes(zlib, n):
    refused(zlib, lambda: verify(zlib, n=n), zlib.ZSAA_ERR_UNSUPPORTED)


def test_verify_workspace_needs_no_device(zlib):
    n = zlib.zsaa_op_draft_verify_workspace(4, 3, 1000)
    assert n > 0 and zlib.zsaa_op_draft_verify_workspace(3, 2, 900) <= n
    refused(zlib, lambda: verify(zlib, ws_bytes=n - 1))
    assert zlib.lib().zsaa_op_draft_verify_workspace(1, 1, 1, None) == zlib.ZSAA_ERR_INVALID_ARG
    refused(zlib, lambda: verify(zlib, dtype=zlib.ZSAA_BF16, target=A + 1))
    refused(zlib, lambda: verify(zlib, dtype=zlib.ZSAA_BF16, target=A + 2, draft=B + 2, ws_bytes=1))  # (2-byte rows are fine)


def test_the_binding_refuses_tensors_of_another_kind(zlib):
    import torch
    host = torch.zeros(4096, dtype=torch.int32)
    refused(zlib, lambda: resize(zlib, refs=host))
    refused(zlib, lambda: fork(zlib, parent=host))
    refused(zlib, lambda: compact(zlib, keep=host))
    refused(zlib, lambda: verify(zlib, target=torch.zeros(4, 4, 1000)))
    refused(zlib, lambda: verify(zlib, uniform=torch.zeros(16, dtype=torch.float64)))


def test_plain_forms_agree_with_closed_ones():
    """The oracle itself: pages come and go, and verified tokens have the target's distribution."""
    refs, table = np.zeros(6, int), np.full((2, 4), -1)
    lens, left = P.resize(refs, 16, table, [0, 0], [33, 16])
    assert lens.tolist() == [33, 16] and table[:, :3].tolist() == [[0, 1, 2], [3, -1, -1]] and left == 2
    lens, left = P.resize(refs, 16, table, lens, [16, 64])
    assert lens.tolist() == [16, 64] and table[1].tolist() == [3, 1, 2, 4] and left == 1 and refs.tolist() == [1, 1, 1, 1, 1, 0]
    lens, left = P.resize(refs, 16, table, lens, [64, 65 - 1])
    assert lens.tolist() == [32, 64] and left == 0
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((2, 1, 6, 1, 16, 2))
    refs, out = np.array([1, 1, 0, 0, 0, 0]), np.full((2, 2), -1)
    old = k.copy()
    lens, left = P.fork(k, v, refs, 16, np.array([[0, 1]]), [20], [0, 0], [20, 16], out)
    assert lens.tolist() == [20, 16] and out.tolist() == [[0, 2], [0, -1]] and refs.tolist() == [3, 1, 1, 0, 0, 0] and left == 3
    assert np.array_equal(k[0, 2, 0, :4], old[0, 1, 0, :4]) and np.array_equal(k[0, 2, 0, 4:], old[0, 2, 0, 4:])
    assert P.compact(k, v, 16, np.array([[0, 1]]), [1], np.array([[3, 17]]), [2], np.array([[0, 1]])).tolist() == [3]
    assert np.array_equal(k[0, 0, 0, 2], old[0, 1, 0, 1]) and np.array_equal(k[0, 0, 0, 1], old[0, 0, 0, 3])

    # over a grid of both numbers and all drafts, tokens appear as often as the target has them
    target, draft = np.log([[[0.5, 0.2, 0.3], [0.2, 0.3, 0.5]]]), np.log([[[0.2, 0.6, 0.2]]])
    count, m = np.zeros(3), 50
    for x, q in enumerate((0.2, 0.6, 0.2)):
        for a in range(m):
            for b in range(m):
                u = np.array([[(a + 0.5) / m, (b + 0.5) / m]])
                acc, tok, lp, _, _ = P.verify(target, draft, np.array([[x]]), None, u)
                count[tok[0, 0]] += q / m / m
                assert acc[0] == (tok[0, 1] >= 0)
    np.testing.assert_allclose(count, [0.5, 0.2, 0.3], atol=0.02)
    acc, tok, lp, _, _ = P.verify(target, None, np.array([[2]]), np.array([0.0]), np.array([[0.9, 0.9]]))
    assert acc[0] == 0 and tok.tolist() == [[0, -1]] and lp[0, 0] == 0
