"""Refusals of the 8-bit cache's calls that need no GPU."""
import os
import subprocess
import sys

import pytest
import torch

from test_quant_cpu import _cache, _fake, built  # noqa: F401  (built: the libraries are there)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


# ------------------------------------------------------------------------------------------- a binding without its extension
_WITHOUT = """
import sys, torch
sys.modules["paper_2411_05787_b200._rkv_calls"] = None           # no such extension
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):    # nor what only a torch with CUDA has
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2411_05787_b200 import rkv, runner, synth, harness
assert rkv.lib.rkv_full_attention(None, None, None, None, None, 0, None) == 1
rkv.RopeTable(device="cpu")
c = object.__new__(rkv.Context)
c.device, c._h, c._key = 0, None, (0, 1, 1, 1, 0)
try:
    c.quant_store(None, None, rkv.RkvQuantCache())
except ImportError as e:
    assert "build it first" in str(e)
    print("refused")
"""


def test_bf16_calls_need_no_extension():
    r = subprocess.run([sys.executable, "-c", _WITHOUT], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "refused", r.stderr


@pytest.mark.parametrize("cc", ["false", "no-such-compiler"])
def test_build_goes_on_without_a_host_compiler(monkeypatch, tmp_path, cc):
    from paper_2411_05787_b200 import build
    stale = tmp_path / "_rkv_calls.so"
    stale.write_bytes(b"")
    monkeypatch.setattr(build, "CALLS_LIB", str(stale))
    monkeypatch.setattr(build, "calls_need_build", lambda: True)
    monkeypatch.setenv("CC", cc)
    with pytest.warns(RuntimeWarning, match="extension is not built"):
        assert build.build() == build.LIB
    assert not stale.exists()           # an older one would be called with other arguments
