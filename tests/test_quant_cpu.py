"""8-bit cache: the oracle's pins and the refusals that need no GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import quant_oracle as QO


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2411_05787_b200 import build
    build.build()


def test_grid_and_rounding_match_the_library_type():
    """The oracle's e4m3 grid and rounding against torch's conversion (an independent implementation)."""
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(QO.VALUES, want, equal_nan=True)
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(20000, generator=g) * 2.0 ** e for e in range(-9, 9)])
    x = x[x.abs() <= 448]
    got = QO.encode(x.double().numpy())
    assert np.array_equal(got, x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    mid = (QO._POSITIVE[1:] + QO._POSITIVE[:-1]) / 2          # ties: to the even code
    assert np.array_equal(QO.encode(mid), np.arange(1, 127) - (np.arange(1, 127) % 2))
    assert QO.encode(np.array([math.inf, -math.inf, math.nan])).tolist() == [0x7f] * 3
    # half a step: 2^-4 relative for normal codes
    x = np.abs(x.double().numpy())
    x = x[x >= 2.0 ** -6]
    assert (np.abs(QO.decode(QO.encode(x)) - x) <= 2.0 ** -4 * x).all()


def test_needed_scale():
    for a, s in ((448.0, 1.0), (448.0001, 2.0), (1.75, 2.0 ** -8), (1.7500001, 2.0 ** -7), (0.0, 2.0 ** -126), (3.3895e38, 2.0 ** 120)):
        assert QO.needed(a) == s
        assert a <= 448 * s


def test_store_in_steps_equals_store_at_once_where_nothing_falls_below_the_grid():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 128)) * np.exp2(rng.integers(0, 3, (200, 1)))
    x = np.where(np.abs(x) < 0.05, 0.05, x)        # above the subnormal codes whatever the block's scale
    once = np.zeros((256, 128), np.uint8), np.ones(4)
    step = np.zeros((256, 128), np.uint8), np.ones(4)
    QO.store(*once, x, 0, 200)
    at = 0
    for n in (1, 62, 1, 1, 64, 71):
        at = QO.store(*step, x[at: at + n], at, n)
    assert at == 200 and np.array_equal(once[0], step[0]) and np.array_equal(once[1], step[1])


def _fake(n_seq=2, n_q=8, n_kv=2):
    """A context without a library handle: the binding's own checks come before any call."""
    from paper_2411_05787_b200 import rkv
    c = object.__new__(rkv.Context)
    c.cfg = rkv.RkvConfig(n_seq, n_q, n_kv, 128, 256, 64, 0, 1, 0.0)
    c.device, c._h, c._key = 0, None, (0, n_seq, n_q, n_kv, 0)
    return rkv, c


def _cache(rkv, n_seq=2, device=0):
    c = rkv.RkvQuantCache()
    c.device, c.n_seq = device, n_seq
    return c


def test_null_and_foreign_arguments_are_refused():
    from paper_2411_05787_b200 import rkv
    L = rkv.lib
    q = rkv.RkvQuantCache()
    assert L.rkv_quant_store(None, None, 0, 0, None, 0, 0, 1, None, None, None, None) == 1
    assert L.rkv_quant_full_attention(None, None, ctypes.byref(q), None, None, 1, 0, None) == 1
    assert L.rkv_quant_score_keys(None, None, ctypes.byref(q), None, 1, None, None, 0, None, None) == 1
    assert L.rkv_quant_select_topk(None, None, ctypes.byref(q), None, 1, None, None, 0, None, None, None) == 1
    assert L.rkv_quant_full_step(None, None, ctypes.byref(q), None, 1, None, None, None, 0, None, None, 0, None) == 1
    assert L.rkv_quant_gather_small(None, None, None, 1, ctypes.byref(q), None, None, None) == 1
    with pytest.raises(ctypes.ArgumentError):    # an 8-bit cache is no bf16 cache
        L.rkv_full_attention(None, None, ctypes.byref(q), None, None, 0, None)


def test_cache_struct_refuses_wrong_tensors():
    from paper_2411_05787_b200 import rkv
    k = torch.zeros((128, 128), dtype=torch.uint8)
    s = torch.ones(2)
    off, cap, n = torch.zeros(1, dtype=torch.int64), torch.full((1,), 128, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    bad = [(k.float(), k, s, s, off, cap, n), (k[:100], k[:100], s, s, off, cap, n), (k, k[:64], s, s, off, cap, n),
           (k, k, s[:1], s, off, cap, n), (k, k, s.double(), s, off, cap, n), (k, k, s, s, off.int(), cap, n),
           (k, k, s, s, off, cap.long(), n)]
    for args in bad:
        with pytest.raises(ValueError):
            rkv.quant_cache_struct(*args)


@pytest.mark.parametrize("what", ["dtype", "heads", "rank", "batch", "host", "count", "sizes"])
def test_store_refuses(what):
    rkv, ctx = _fake()
    k = torch.zeros((2, 3, 2, 128), dtype=torch.bfloat16)
    v, kw = k, {}
    if what == "dtype":
        k = k.float()
    elif what == "heads":
        k = torch.zeros((2, 3, 4, 128), dtype=torch.bfloat16)
    elif what == "rank":
        k = k[0]
    elif what == "batch":
        k = k[:1]
    elif what == "sizes":
        v = torch.zeros((2, 2, 2, 128), dtype=torch.bfloat16)
    elif what == "count":
        kw = dict(count=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):      # ("host": tensors of the CPU)
        ctx.quant_store(k, v, _cache(rkv), **kw)


def test_attention_and_rebuild_refuse():
    rkv, ctx = _fake()
    q = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ctx.quant_full_attention(q.float(), _cache(rkv), q)
    with pytest.raises(ValueError):
        ctx.quant_full_attention(q[:1], _cache(rkv), q)
    with pytest.raises(ValueError):
        ctx.quant_full_attention(q, _cache(rkv), q, active=torch.ones(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        ctx.quant_full_attention(q, _cache(rkv, device=1), q)
    with pytest.raises(ValueError):
        ctx.quant_full_attention(q, _cache(rkv, n_seq=3), q)
    idx = torch.zeros((2, 2, 4), dtype=torch.int32)
    with pytest.raises(ValueError):
        ctx.quant_gather_small(idx, torch.zeros(2, dtype=torch.int32), 5, _cache(rkv), rkv.RkvCache())
    with pytest.raises(ValueError):
        ctx.quant_gather_small(idx.long(), torch.zeros(2, dtype=torch.int32), 4, _cache(rkv), rkv.RkvCache())


def test_extension_refuses_wrong_kinds():
    """What is no tensor, no cache of the right class, no context's key."""
    rkv, ctx = _fake()
    q = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        ctx.quant_full_attention(q, rkv.RkvCache(), q)
    with pytest.raises(TypeError):
        ctx.quant_gather_small(torch.zeros((2, 2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 4, _cache(rkv), _cache(rkv))
    with pytest.raises(ValueError):
        ctx.quant_full_attention(None, _cache(rkv), q)
    with pytest.raises(AttributeError):
        ctx.quant_full_attention([1, 2], _cache(rkv), q)
    with pytest.raises(TypeError):
        rkv._calls.quant_store(ctx._key)
    with pytest.raises(TypeError):
        rkv._calls.quant_store((0, 1), q, q, _cache(rkv), None, None, None)
    idx, ks = torch.zeros((2, 2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        ctx.quant_gather_small(idx, ks, "4", _cache(rkv), rkv.RkvCache())
    with pytest.raises(ValueError):
        ctx.quant_gather_small(idx, ks, 1 << 40, _cache(rkv), rkv.RkvCache())


def test_another_current_device_and_a_closed_context(monkeypatch):
    """The library refuses to launch while another device is current: the call is made again on the context's own; a
    refusal there, or of a closed context, is an error."""
    import contextlib
    rkv, ctx = _fake()
    ctx._key, ctx.device = (1,) + ctx._key[1:4] + (1,), 1
    made, on = [], []

    @contextlib.contextmanager
    def device(i):
        on.append(i)
        yield
        on.pop()

    monkeypatch.setattr(rkv, "_current_device", lambda: on[-1] if on else 0)
    monkeypatch.setattr(torch.cuda, "device", device)

    def call(rc_there):
        def f(*args):
            made.append((args, list(on)))
            return rc_there if on else 1
        return f

    ctx._done(call(0)(7), call(0), 7)
    assert made == [((7,), []), ((7,), [1])] and not on
    with pytest.raises(rkv.RkvError):
        ctx._done(1, call(1), 7)
    made.clear()
    ctx._key = (0,) + ctx._key[1:]
    with pytest.raises(rkv.RkvError):
        ctx._done(1, call(0), 7)
    assert not made
