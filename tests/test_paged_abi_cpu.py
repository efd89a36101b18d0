"""Argument checks of the paged-cache and beam-search calls: refused on the host,
before any device work (the addresses below are never dereferenced)."""

import ctypes as C

import numpy as np
import pytest

import paged_ref as R

A = 1 << 20
FAR = 1 << 40


def pages(z, **kw):
    f = dict(k=A, v=FAR, n_pages=64, page_size=16, n_kv_heads=2, head_dim=64, dtype=z.ZSAA_BF16)
    f.update(kw)
    return z.zsaa_pages(*f.values())


def refused(z, call, status=None):
    with pytest.raises(z.ZsaaError) as e:
        call()
    assert e.value.status == (z.ZSAA_ERR_INVALID_ARG if status is None else status), str(e.value)


BAD_PAGES = [dict(k=None), dict(v=None), dict(k=A + 8), dict(n_pages=0), dict(n_kv_heads=0), dict(dtype=7),
             dict(n_pages=1 << 30)]
UNSUPPORTED_PAGES = [dict(page_size=0), dict(page_size=8), dict(page_size=24), dict(page_size=512),
                     dict(head_dim=32), dict(head_dim=96), dict(head_dim=256)]


def append(z, kv=None, **kw):
    f = dict(qkv=A, ld=512, qkv_dtype=z.ZSAA_BF16, T=4, Hq=4, pos=A, theta=1e4, cu=A, S=2, table=A, cols=3, lens=A,
             q_out=FAR)
    f.update(kw)
    z.zsaa_op_paged_append(kv or pages(z), *f.values(), stream=0)


def attention(z, kv=None, **kw):
    f = dict(q=A, S=4, n_q=1, Hq=4, table=A, cols=3, lens=A, cu=A, G=2, ptable=A, pcols=5, plens=A, out=FAR, lse=A,
             ws=FAR, ws_bytes=1 << 40)
    f.update(kw)
    z.zsaa_op_paged_attention(kv or pages(z), *f.values(), stream=0)


def select(z, **kw):
    f = dict(logits=A, ld=1000, B=2, W=4, V=1000, scores=A, done=A, eos=2, K=4, scores_out=FAR, parent=A, token=A,
             done_out=FAR, ws=A, ws_bytes=1 << 40)
    f.update(kw)
    z.zsaa_op_beam_select(*f.values(), stream=0)


def reorder(z, layers=None, **kw):
    f = dict(B=2, W=4, K=4, parent=A, table=A, table_out=FAR, cols=5, lens=A, lens_out=FAR, fresh=A)
    f.update(kw)
    layers = layers or [pages(z), pages(z)]
    z.zsaa_op_beam_reorder((z.zsaa_pages * len(layers))(*layers), *f.values(), stream=0)


@pytest.mark.parametrize("kw", BAD_PAGES + UNSUPPORTED_PAGES)
def test_pools_are_checked_by_every_call(zlib, kw):
    st = zlib.ZSAA_ERR_UNSUPPORTED if kw in UNSUPPORTED_PAGES else None
    refused(zlib, lambda: append(zlib, pages(zlib, **kw)), st)
    refused(zlib, lambda: attention(zlib, pages(zlib, **kw)), st)
    refused(zlib, lambda: reorder(zlib, [pages(zlib), pages(zlib, **kw)]), st)


@pytest.mark.parametrize("kw", [
    dict(qkv=None), dict(pos=None), dict(table=None), dict(lens=None), dict(T=0), dict(S=0), dict(Hq=0), dict(Hq=3),
    dict(cu=None), dict(qkv_dtype=5), dict(theta=0.5), dict(theta=float("inf")), dict(theta=float("nan")), dict(cols=0),
    dict(cols=1 << 28), dict(ld=511), dict(ld=516), dict(qkv=A + 2), dict(q_out=FAR + 8), dict(q_out=A + 64), dict(ld=-8),
    dict(pos=A + 2), dict(cu=A + 1), dict(table=A + 2), dict(lens=A + 3)])
def test_append_refusals(zlib, kw):
    refused(zlib, lambda: append(zlib, **kw))


def test_append_refuses_bf16_rows_for_a_float32_pool(zlib):
    kv = pages(zlib, dtype=zlib.ZSAA_F32)
    refused(zlib, lambda: append(zlib, kv, qkv_dtype=zlib.ZSAA_BF16))


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(table=None), dict(lens=None), dict(out=None), dict(ws=None), dict(S=0), dict(Hq=0), dict(Hq=5),
    dict(G=-1), dict(cols=0), dict(pcols=0), dict(cu=None), dict(ptable=None), dict(plens=None), dict(q=A + 8),
    dict(out=FAR + 2), dict(ws=FAR + 8), dict(ws_bytes=64), dict(out=A + 256), dict(S=1 << 30), dict(G=1 << 30),
    dict(cols=1 << 26, S=1 << 20), dict(Hq=1 << 17),
    dict(table=A + 2), dict(lens=A + 1), dict(lse=A + 2), dict(cu=A + 2), dict(ptable=A + 2), dict(plens=A + 2)])
def test_attention_refusals(zlib, kw):
    refused(zlib, lambda: attention(zlib, **kw))


@pytest.mark.parametrize("n_q", [0, 17])
def test_attention_refuses_more_new_entries_than_it_takes(zlib, n_q):
    refused(zlib, lambda: attention(zlib, n_q=n_q), zlib.ZSAA_ERR_UNSUPPORTED)


def test_attention_workspace_needs_no_device_and_covers_smaller_calls(zlib):
    kv = pages(zlib)
    n = zlib.zsaa_op_paged_attention_workspace(kv, 8, 1, 4, 2, 10, 20)
    assert n > 0
    assert zlib.zsaa_op_paged_attention_workspace(kv, 8, 1, 4, 0, 10, 0) <= n
    assert zlib.zsaa_op_paged_attention_workspace(kv, 8, 1, 4, 0, 10, -5) <= n  # not looked at without groups
    assert zlib.zsaa_op_paged_attention_workspace(kv, 4, 1, 4, 2, 10, 20) <= n
    refused(zlib, lambda: attention(zlib, S=8, ws_bytes=n - 1, cols=10, pcols=20))
    assert zlib.lib().zsaa_op_paged_attention_workspace(None, 1, 1, 1, 0, 1, 0, None) == zlib.ZSAA_ERR_INVALID_ARG


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_attention_refuses_rows_whose_blocks_pass_31_bits(zlib, page):
    """Entries are walked in blocks of up to 128 keys, and the numbers of a row's last block
    still have to fit an int32."""
    kv = pages(zlib, page_size=page, n_kv_heads=1)
    most = (2 ** 31 - 256) // page
    for dtype in (zlib.ZSAA_BF16, zlib.ZSAA_F32):
        kv.dtype = dtype
        assert zlib.zsaa_op_paged_attention_workspace(kv, 1, 1, 1, 0, most, 0) > 0
        assert zlib.zsaa_op_paged_attention_workspace(kv, 1, 1, 1, 1, 1, most) > 0
        for cols in range(most + 1, (2 ** 31 - 1) // page + 2):
            refused(zlib, lambda: zlib.zsaa_op_paged_attention_workspace(kv, 1, 1, 1, 0, cols, 0))
            refused(zlib, lambda: zlib.zsaa_op_paged_attention_workspace(kv, 1, 1, 1, 1, 1, cols))
            refused(zlib, lambda: attention(zlib, kv, cols=cols, Hq=1))
            refused(zlib, lambda: attention(zlib, kv, pcols=cols, Hq=1))


@pytest.mark.parametrize("kw", [
    dict(logits=None), dict(scores_out=None), dict(parent=None), dict(token=None), dict(ws=None), dict(B=0), dict(W=0),
    dict(W=65), dict(V=0), dict(V=(1 << 26) + 1, ld=1 << 27), dict(K=0), dict(K=65), dict(V=3, W=1, K=4, eos=1),
    dict(ld=999), dict(logits=A + 2), dict(eos=-2), dict(eos=1000), dict(eos=-1), dict(ws=A + 8), dict(ws_bytes=100),
    dict(scores_out=A + 16), dict(done_out=A + 4), dict(B=1 << 26),
    dict(scores=A + 2), dict(scores_out=FAR + 1), dict(parent=A + 2), dict(token=A + 2)])
def test_select_refusals(zlib, kw):
    refused(zlib, lambda: select(zlib, **kw))


def test_select_workspace(zlib):
    n = zlib.zsaa_op_beam_select_workspace(2, 4, 1000, 4)
    refused(zlib, lambda: select(zlib, ws_bytes=n - 1))
    refused(zlib, lambda: zlib.zsaa_op_beam_select_workspace(2, 4, 1000, 0))
    assert zlib.lib().zsaa_op_beam_select_workspace(1, 1, 1, 1, None) == zlib.ZSAA_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(parent=None), dict(table=None), dict(table_out=None), dict(lens=None), dict(lens_out=None), dict(fresh=None),
    dict(B=0), dict(W=0), dict(W=65), dict(K=0), dict(K=65), dict(cols=0), dict(table_out=A + 4), dict(lens_out=A + 4),
    dict(parent=A + 2), dict(table=A + 2), dict(table_out=FAR + 2), dict(lens=A + 2), dict(lens_out=FAR + 2), dict(fresh=A + 2)])
def test_reorder_refusals(zlib, kw):
    refused(zlib, lambda: reorder(zlib, **kw))


def test_reorder_refuses_unlike_layers_and_their_number(zlib):
    for kw in (dict(n_pages=65), dict(page_size=32), dict(n_kv_heads=1), dict(head_dim=128),
               dict(head_dim=64, dtype=zlib.ZSAA_F32)):
        refused(zlib, lambda: reorder(zlib, [pages(zlib), pages(zlib, **kw)]))
    refused(zlib, lambda: reorder(zlib, [pages(zlib)] * 65))
    L = zlib.lib()
    assert L.zsaa_op_beam_reorder(None, 1, 1, 1, 1, A, A, FAR, 1, A, FAR, A, None) == zlib.ZSAA_ERR_INVALID_ARG
    one = pages(zlib)
    assert L.zsaa_op_beam_reorder(C.addressof(one), 0, 1, 1, 1, A, A, FAR, 1, A, FAR, A, None) == zlib.ZSAA_ERR_INVALID_ARG


def test_the_binding_refuses_tensors_of_another_kind(zlib):
    import torch
    host = torch.zeros(64, dtype=torch.int32)
    refused(zlib, lambda: append(zlib, pos=host))
    refused(zlib, lambda: select(zlib, logits=torch.zeros(8, 1000)))
    refused(zlib, lambda: zlib.make_pages(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64)))
    refused(zlib, lambda: zlib.make_pages_list([], []))


@pytest.mark.parametrize("flags", [[0] * 8, np.zeros(8, np.uint8), np.zeros(8, bool), "01010101", (0, 1)])
@pytest.mark.parametrize("name", ["done", "done_out"])
def test_the_binding_refuses_flags_that_are_no_tensor(zlib, name, flags):
    refused(zlib, lambda: select(zlib, **{name: flags}))


@pytest.mark.parametrize("dtype", ["int8", "int32", "float32", "uint8", "bool"])
def test_the_binding_refuses_flags_of_other_types_or_on_the_host(zlib, dtype):
    import torch
    for name in ("done", "done_out"):
        refused(zlib, lambda: select(zlib, **{name: torch.zeros(8, dtype=getattr(torch, dtype))}))


def test_plain_forms_agree_with_closed_ones():
    """The oracle itself: one key gives its value, equal keys the mean, a rotation keeps
    scores relative, and selection orders ties as stated."""
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((2, 3, 1, 16, 32))
    q = rng.standard_normal((1, 1, 2, 32))
    out, lse = R.attention(k[:, :], v, q, [[2]], [1])
    np.testing.assert_allclose(out[0, 0, 0], v[2, 0, 0])
    k[1] = k[1, :, :1]
    out, lse = R.attention(k, v, q, [[0]], [0], groups=[0, 1], ptable=[[1]], plens=[5])
    np.testing.assert_allclose(out[0, 0, 1], v[1, 0, :5].mean(0))
    np.testing.assert_allclose(lse[0, 0, 1], (q[0, 0, 1] @ k[1, 0, 0]) / np.sqrt(32) / np.log(2) + np.log2(5))
    x, y = rng.standard_normal((2, 32))
    np.testing.assert_allclose(R.rope(x, 7, 1e4) @ R.rope(y, 3, 1e4), R.rope(x, 104, 1e4) @ R.rope(y, 100, 1e4))
    s, par, tok, ended, _ = R.select(np.zeros((1, 2, 4), np.float32), np.zeros((1, 2), np.float32), None, 1, 6)
    assert par.tolist() == [[0, 0, 0, 0, 1, 1]] and tok.tolist() == [[0, 1, 2, 3, 0, 1]]
    np.testing.assert_allclose(s, -np.log(4.0))
    assert ended.tolist() == [[False, True, False, False, False, True]]
    s, par, tok, ended, _ = R.select(np.array([[[np.nan, 1, 2], [0, -np.inf, 5]]], np.float32), None, None, -1, 6)
    assert par.tolist() == [[1, 1, 1, 0, 0, 0]] and tok.tolist() == [[2, 0, 1, 2, 1, 0]]
