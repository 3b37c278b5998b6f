"""Refusals of the 8-bit cache's calls that need no GPU."""
import pytest
import torch

from test_quant_cpu import _cache, _fake, built  # noqa: F401  (built: the libraries are there)


def _small(rkv, n_seq, device=0):
    c = rkv.RkvCache()
    c.device, c.n_seq = device, n_seq
    return c


@pytest.mark.parametrize("what", ["device", "several devices", "sequences", "undescribed"])
def test_rebuild_refuses_a_small_cache_that_does_not_fit(what):
    """The kernel reads row_offset and cap for every sequence of the context and writes where they say."""
    rkv, ctx = _fake()
    small = {"device": lambda: _small(rkv, 2, 1), "several devices": lambda: _small(rkv, 2, -1), "sequences": lambda: _small(rkv, 1),
             "undescribed": rkv.RkvCache}[what]()
    idx, ks = torch.zeros((2, 2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="small cache"):
        ctx.quant_gather_small(idx, ks, 4, _cache(rkv), small)
    with pytest.raises(ValueError, match="topk_idx"):     # one that fits: the next argument is looked at
        ctx.quant_gather_small(idx, ks, 4, _cache(rkv), _small(rkv, 3))


def test_struct_arrays_of_different_length_count_as_the_shortest(monkeypatch):
    from paper_2411_05787_b200 import rkv
    monkeypatch.setattr(rkv, "_ptr", lambda t: t.data_ptr())
    k = torch.zeros((64, 128), dtype=torch.bfloat16)
    for sizes in ((1, 2, 2), (2, 1, 2), (2, 2, 1)):
        off, cap, n = (torch.zeros(s, dtype=d) for s, d in zip(sizes, (torch.int64, torch.int32, torch.int32)))
        assert rkv.cache_struct(k, k, off, cap, n).n_seq == 1
    off, cap, n = (torch.zeros(2, dtype=d) for d in (torch.int64, torch.int32, torch.int32))
    assert rkv.cache_struct(k, k, off, cap.to("meta"), n).device == -1
