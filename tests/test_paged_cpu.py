"""The paged cache without a GPU: the oracle's pins, and what the binding and the library refuse."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from test_quant_cpu import _fake, built  # noqa: F401  (built: the libraries are there)

pytestmark = pytest.mark.usefixtures("built")


# ----------------------------------------------------------------------------------------------------------- the oracle
def test_rows_come_from_their_pages():
    pool = np.arange(5 * 2 * 4 * 3).reshape(5, 2, 4, 3)
    table = [3, 0, 4]
    got = PO.rows(pool, table, 4, 10)
    for p in range(10):
        page, r = PO.place(table, 4, p)
        assert np.array_equal(got[:, p], pool[page, :, r])


def test_no_key_of_a_page_exceeds_its_score():
    g = np.random.default_rng(1)
    k, q = g.normal(size=(6, 16, 128)), g.normal(size=(3, 128))
    s = PO.scores(q, k.min(1), k.max(1))
    assert (np.einsum("hc,prc->phr", q, k).max((1, 2)) <= s).all()
    same = np.repeat(k[:, :1], 16, 1)                      # pages of one key: the score is the product
    assert np.allclose(PO.scores(q, same.min(1), same.max(1)), (k[:, 0] @ q.T).max(1))


def test_selection_order():
    s = np.array([0.0, 5.0, 7.0, 5.0, 1.0, 9.0, 0.0])
    assert PO.select(s, 3, 0, 0) == [1, 2, 5]              # the lower of two equal scores
    assert PO.select(s, 4, 1, 1) == [0, 2, 5, 6]
    assert PO.select(s, 2, 2, 1) == [0, 1]                 # forced pages tie too
    assert PO.select(s, 9, 1, 1) == list(range(7))


def test_bounds_join_or_begin_anew():
    new = np.array([[1.0, np.nan], [3.0, -2.0]])
    lo, hi = PO.bounds_after(np.array([0.0, -5.0]), np.array([2.0, 5.0]), new, True)
    assert lo.tolist() == [0.0, -5.0] and hi.tolist() == [3.0, 5.0]
    lo, hi = PO.bounds_after(np.array([0.0, -5.0]), np.array([2.0, 5.0]), new, False)
    assert lo.tolist() == [1.0, -2.0] and hi.tolist() == [3.0, -2.0]


def test_attention_over_all_pages_is_attention():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((8, 128), (2, 40, 128), (2, 40, 128)))
    want = torch.nn.functional.scaled_dot_product_attention(q[None, :, None], k[None], v[None], enable_gqa=True)[0, :, 0]
    out, _ = PO.attend(q.numpy(), k.numpy(), v.numpy())
    assert np.allclose(out, want.numpy())
    some = [np.arange(0, 40, 2), np.arange(5)]
    out, _ = PO.attend(q.numpy(), k.numpy(), v.numpy(), some)
    for i, at in enumerate(some):
        part, _ = PO.attend(q.numpy()[4 * i: 4 * i + 4], k.numpy()[i: i + 1, at], v.numpy()[i: i + 1, at])
        assert np.allclose(out[4 * i: 4 * i + 4], part)


# ------------------------------------------------------------------------------------------------------------- refusals
def _cache(rkv, n_seq=2, device=0, n_kv=2, bounds=True):
    c = rkv.RkvPagedCache(0, 0, 16 if bounds else 0, 16 if bounds else 0, 4, 16, 3, 0, 0)
    c.device, c.n_seq, c.n_kv = device, n_seq, n_kv
    return c


def test_null_and_foreign_arguments_are_refused():
    from paper_2411_05787_b200 import rkv
    L, c = rkv.lib, rkv.RkvPagedCache()
    assert L.rkv_paged_append(None, None, 1, 0, 0, 1, None, None, None, 0, 0, 1.0, ctypes.byref(c), None, None) == 1
    assert L.rkv_paged_attention(None, None, ctypes.byref(c), None, None, 0, None, 0, None) == 1
    assert L.rkv_paged_sparse_attention(None, None, ctypes.byref(c), None, 1, 0, 0, None, None, 0, None) == 1
    with pytest.raises(ctypes.ArgumentError):
        L.rkv_full_attention(None, None, ctypes.byref(c), None, None, 0, None)


@pytest.mark.parametrize("what", ["page", "rank", "dtype", "channels", "values", "one bound", "bounds", "table", "table rank",
                                  "length", "length type", "host", "contiguous"])
def test_cache_struct_refuses_wrong_tensors(what, monkeypatch):
    from paper_2411_05787_b200 import rkv
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    v, lo, hi = k.clone(), torch.zeros((4, 2, 128), dtype=torch.bfloat16), torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    table, n = torch.zeros((3, 5), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    if what == "page":
        k = v = torch.zeros((4, 2, 48, 128), dtype=torch.bfloat16)
    elif what == "rank":
        k = k[0]
    elif what == "dtype":
        k = k.half()
    elif what == "channels":
        k = v = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    elif what == "values":
        v = v[:2]
    elif what == "one bound":
        hi = None
    elif what == "bounds":
        hi = hi[:2]
    elif what == "table":
        table = table.long()
    elif what == "table rank":
        table = table[0]
    elif what == "length":
        n = n[:2]
    elif what == "length type":
        n = n.long()
    elif what == "contiguous":
        monkeypatch.setattr(torch.Tensor, "is_cuda", True)
        k = v = torch.zeros((4, 16, 2, 128), dtype=torch.bfloat16).transpose(1, 2)
    with pytest.raises(ValueError):          # ("host": tensors of the CPU)
        rkv.paged_cache_struct(k, v, table, n, lo, hi)


@pytest.mark.parametrize("what", ["dtype", "width", "batch", "rank", "device", "sequences", "heads", "foreign", "table"])
def test_append_refuses(what):
    rkv, ctx = _fake()
    x = torch.zeros((2, 3, 12 * 128), dtype=torch.bfloat16)
    q = torch.zeros((2, 3, 8, 128), dtype=torch.bfloat16)
    c, table, err = _cache(rkv), None, ValueError
    if what == "dtype":
        x = x.half()
    elif what == "width":
        x = x[..., : 11 * 128]
    elif what == "batch":
        x = x[:1]
    elif what == "rank":
        x = x[0]
    elif what == "device":
        c = _cache(rkv, device=1)
    elif what == "sequences":
        c = _cache(rkv, n_seq=3)
    elif what == "heads":
        c = _cache(rkv, n_kv=4)
    elif what == "foreign":
        c, err = rkv.RkvQuantCache(), TypeError
    elif what == "table":
        table, err = object(), (TypeError, ValueError)
    with pytest.raises(err):
        ctx.paged_append(x, c, table, q)


def test_attention_refuses():
    rkv, ctx = _fake()
    q = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    idx = torch.zeros((2, 2, 3), dtype=torch.int32)
    for bad in (q.float(), q[:1], q.transpose(0, 1)):
        with pytest.raises(ValueError):
            ctx.paged_attention(bad, _cache(rkv), q)
        with pytest.raises(ValueError):
            ctx.paged_sparse_attention(bad, _cache(rkv), 3, idx, q)
    with pytest.raises(ValueError):
        ctx.paged_attention(q, _cache(rkv, n_seq=1), q)
    with pytest.raises(TypeError):
        ctx.paged_sparse_attention(q, rkv.RkvCache(), 3, idx, q)


def test_alloc_of_paged_caches():
    from paper_2411_05787_b200 import synth
    for rooms, shared in (([100], 8), ([100, 20], 32)):
        with pytest.raises(ValueError):
            synth.alloc_paged_cache(rooms, 1, 16, "cpu", shared=shared)
    c = synth.alloc_paged_cache([100, 40], 2, 16, "cpu", shared=32)
    assert c.table.tolist() == [[0, 1, 2, 3, 4, 5, 6], [0, 1, 7, -1, -1, -1, -1]] and c.k.shape == (8, 2, 16, 128)
    assert c.shared.tolist() == [0, 1] and c.page == 16
