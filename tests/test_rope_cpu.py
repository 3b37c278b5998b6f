"""Rotary positions: the host's frequencies against the oracle, and the refusals that need no GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import quant_oracle as QO


@pytest.fixture(scope="module")
def rkv():
    from paper_2411_05787_b200 import build
    build.build()
    from paper_2411_05787_b200 import rkv
    return rkv


CASES = [dict(), dict(rot_dim=64, theta=500000.0), dict(rot_dim=16, theta=10000.0, scaling="linear", factor=4.0),
         dict(theta=500000.0, scaling="bands", factor=8.0, trained_len=8192, low=1.0, high=4.0),
         dict(rot_dim=96, theta=1e6, scaling="bands", factor=32.0, trained_len=4096, low=1.0, high=2.0),
         dict(theta=1e6, scaling="ramp", factor=4.0, trained_len=32768),
         dict(rot_dim=48, theta=10000.0, scaling="ramp", factor=40.0, trained_len=4096, fast=16.0, slow=2.0),
         dict(rot_dim=32, theta=2.0, scaling="ramp", factor=2.0, trained_len=1)]


@pytest.mark.parametrize("kw", CASES)
def test_frequencies(rkv, kw):
    t = rkv.RopeTable(device="cpu", **kw)
    rot = kw.get("rot_dim", 128)
    names = dict(scaling="none", factor=1.0, trained_len=8192, low=1.0, high=4.0, fast=32.0, slow=1.0)
    f, amp = QO.rope_frequencies(rot, kw.get("theta", 10000.0), **{n: kw.get(n, v) for n, v in names.items()})
    assert len(t.turns) == rot // 2 and t.rot_dim == rot
    got = np.array([x / 2.0 ** 64 for x in t.turns]) * 2 * math.pi
    assert np.allclose(got, f, rtol=1e-14, atol=2.0 ** -62)
    assert t.amplitude == np.float32(amp)
    assert [x & (2 ** 64 - 1) for x in t.freqs.tolist()] == t.turns


def test_bands_and_ramp_meet_the_unscaled_ends(rkv):
    """Fast pairs are left alone and slow ones divided by the factor, as linear scaling divides all."""
    plain = rkv.RopeTable(theta=500000.0, device="cpu").turns
    linear = rkv.RopeTable(theta=500000.0, scaling="linear", factor=8.0, device="cpu").turns
    for how in ("bands", "ramp"):
        t = rkv.RopeTable(theta=500000.0, scaling=how, factor=8.0, device="cpu").turns
        assert t[0] == plain[0] and t[-1] == linear[-1]
        assert all(a <= b <= c for a, b, c in zip(linear, t, plain))
        assert any(a < b < c for a, b, c in zip(linear, t, plain))


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144), dict(theta=1.0), dict(theta=math.inf),
                                dict(theta=math.nan), dict(scaling="linear", factor=0.5), dict(scaling="bands", factor=math.nan),
                                dict(scaling="bands", trained_len=0), dict(scaling="bands", low=4.0, high=4.0),
                                dict(scaling="ramp", fast=1.0, slow=1.0), dict(scaling="ramp", slow=0.0)])
def test_tables_refused(rkv, kw):
    with pytest.raises(rkv.RkvError):
        rkv.RopeTable(device="cpu", **kw)


def test_unknown_names_are_refused(rkv):
    with pytest.raises(ValueError):
        rkv.RopeTable(layout="third", device="cpu")
    with pytest.raises(ValueError):
        rkv.RopeTable(scaling="other", device="cpu")
    assert rkv.lib.rkv_rope_frequencies(None, None, None) == 1
    assert rkv.lib.rkv_rope(None, None, 1, 0, None, 1, 1, 1, None, 128, 0, 1.0, None, None, None, None) == 1


def test_call_refusals(rkv):
    ctx = object.__new__(rkv.Context)
    ctx.cfg = rkv.RkvConfig(1, 4, 2, 128, 256, 64, 0, 1, 0.0)
    ctx.device, ctx._h, ctx._key = 0, None, (0, 1, 4, 2, 0)
    table = rkv.RopeTable(device="cpu")
    bf = dict(dtype=torch.bfloat16)
    qkv, pos = torch.zeros((3, 8 * 128), **bf), torch.zeros(3, dtype=torch.int32)
    q, k, v = torch.zeros((3, 4, 128), **bf), torch.zeros((3, 2, 128), **bf), torch.zeros((3, 2, 128), **bf)
    for args in ((qkv.half(), pos, table, q, k, v), (qkv[:, :896], pos, table, q, k, v), (qkv.view(-1), pos, table, q, k, v),
                 (qkv, pos.long(), table, q, k, v), (qkv, pos[:2], table, q, k, v), (qkv, pos, table, q.float(), k, v),
                 (qkv, pos, table, q[:2], k, v), (qkv, pos, table, q, q, v), (qkv, pos, table, q, k, q),
                 (qkv, pos, table, q, k, v)):        # (the last: tensors of the CPU)
        with pytest.raises(ValueError):
            ctx.rope(*args)
