"""Rotary positions on the GPU against the fp64 oracle.

Tolerance per element: 2^-8 |want| (half a bf16 step) + 2^-20 amp (|x| + |y|): the angle is off by at most 2^-31 half turns
plus half an fp32 step of at most one (2^-25 pi), sine and cosine by a few 2^-24, the two products and their sum by three
half steps of 2^-24.
"""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as QO

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rkv():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2411_05787_b200 import rkv
    return rkv


def f64(t):
    return t.detach().double().cpu().numpy()


def make(rkv, n, nq, nkv, dtype, seed, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((n, (nq + 2 * nkv) * 128 + pad), generator=g, device="cuda").to(dtype)[:, : (nq + 2 * nkv) * 128]
    out = [torch.full((n + 1, h, 128), 7.0, dtype=torch.bfloat16, device="cuda") for h in (nq, nkv, nkv)]
    return rkv.Context(1, 1, 1, 64, 64), x, out     # (the heads are the tensors')


def check(x, pos, outs, nq, nkv, f, amp, layout):
    n = x.shape[0]
    x = f64(x).reshape(n, nq + 2 * nkv, 128)
    want = np.concatenate([QO.rope(x[:, : nq + nkv], pos, f, amp, layout), x[:, nq + nkv:]], axis=1)
    r = len(f)
    size = np.abs(x).copy()
    i = np.arange(r)
    u, w = (i, i + r) if layout == "half" else (2 * i, 2 * i + 1)
    size[..., u] = size[..., w] = np.abs(x[..., u]) + np.abs(x[..., w])
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * amp * size
    got = np.concatenate([f64(t[:n]) for t in outs], axis=1)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)
    for t in outs:
        assert (t[n:] == 7).all()        # rows behind the last token


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("n", [1, 3, 5, 130])
def test_rope(rkv, n, rot, layout, dtype):
    nq, nkv = (28, 4) if rot != 64 else (3, 1)
    ctx, x, (q, k, v) = make(rkv, n, nq, nkv, dtype, rot + n, pad=64 if n > 1 else 0)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 977 + 100003
    t = rkv.RopeTable(rot, 500000.0, layout)
    ctx.rope(x, pos, t, q[:n], k[:n], v[:n])
    f, amp = QO.rope_frequencies(rot, 500000.0)
    check(x, pos.cpu().numpy(), (q, k, v), nq, nkv, f, amp, layout)
    if dtype == torch.bfloat16:
        assert torch.equal(v[:n].reshape(n, -1), x[:, (nq + nkv) * 128:])
    assert ctx.device_status() == 0


def test_rope_any_heads(rkv):
    for nq, nkv in ((28, 8), (32, 1), (1, 3)):
        ctx, x, (q, k, v) = make(rkv, 6, nq, nkv, torch.bfloat16, nq)
        pos = torch.arange(6, dtype=torch.int32, device="cuda") + 5000
        ctx.rope(x, pos, rkv.RopeTable(80, 10000.0), q[:6], k[:6], v[:6])
        f, amp = QO.rope_frequencies(80, 10000.0)
        check(x, pos.cpu().numpy(), (q, k, v), nq, nkv, f, amp, "half")


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=4.0), dict(scaling="bands", factor=8.0),
                                dict(scaling="ramp", factor=4.0, trained_len=32768)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_scaled(rkv, kw, layout):
    ctx, x, (q, k, v) = make(rkv, 64, 4, 1, torch.float32, 5)
    pos = torch.arange(64, dtype=torch.int32, device="cuda") * 2048
    t = rkv.RopeTable(128, 1e6, layout, **kw)
    ctx.rope(x, pos, t, q[:64], k[:64], v[:64])
    f, amp = QO.rope_frequencies(128, 1e6, **kw)
    check(x, pos.cpu().numpy(), (q, k, v), 4, 1, f, amp, layout)


def test_rope_any_position(rkv):
    """Zero, negative and the largest positions: the angle's fraction of a turn is formed in whole numbers."""
    pos_h = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1 << 20, -12345]
    n = len(pos_h)
    ctx, x, (q, k, v) = make(rkv, n, 2, 1, torch.float32, 6)
    t = rkv.RopeTable(32, 10000.0)
    ctx.rope(x, torch.tensor(pos_h, dtype=torch.int32, device="cuda"), t, q[:n], k[:n], v[:n])
    # the oracle's angle from the table's own turns, in whole numbers, so that 2^31 * theta^(-2i/rot) costs it no bits
    turns = np.array([[((p * f) % (1 << 64)) / 2.0 ** 64 for f in t.turns] for p in pos_h])
    xs = f64(x).reshape(n, 4, 128)
    for i in range(n):
        f = turns[i] * 2 * np.pi
        check(x[i: i + 1], np.ones(1), [torch.cat([o[i: i + 1], torch.full_like(o[:1], 7.0)]) for o in (q, k, v)], 2, 1, f, 1.0, "half")
    assert torch.equal(q[0].float(), x[0, :256].view(2, 128).to(torch.bfloat16).float())     # position 0 turns nothing
    assert xs.shape == (n, 4, 128)


def test_rope_without_values_and_in_place_of_the_loop_s_kernel(rkv):
    """v=None leaves the values alone; one fp32 token, unscaled, half layout is what the decode loop's split computes."""
    from paper_2411_05787_b200 import harness
    ctx, x, (q, k, v) = make(rkv, 1, 32, 8, torch.float32, 9)
    pos = torch.tensor([32801], dtype=torch.int32, device="cuda")
    ctx.rope(x, pos, rkv.RopeTable(128, 500000.0), q[:1], k[:1])
    assert (v == 7).all()
    q2, k2, v2 = torch.empty_like(q[:1]), torch.empty_like(k[:1]), torch.empty_like(v[:1])
    harness.rope_split(x[0].contiguous(), pos, 500000.0, q2, k2, v2, 32, 8)
    assert (q[:1].float() - q2.float()).abs().max() <= 2.0 ** -6 * q.float().abs().max()


def test_rope_captured_on_another_stream(rkv):
    ctx, x, (q, k, v) = make(rkv, 9, 8, 2, torch.bfloat16, 12)
    pos = torch.arange(9, dtype=torch.int32, device="cuda")
    t = rkv.RopeTable(128, 10000.0, "interleaved")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            ctx.rope(x, pos, t, q[:9], k[:9], v[:9])
        pos += 1000
        graph.replay()
    torch.cuda.synchronize()
    f, amp = QO.rope_frequencies(128, 10000.0)
    check(x, pos.cpu().numpy(), (q, k, v), 8, 2, f, amp, "interleaved")


def test_rope_library_refusals(rkv):
    ctx, x, (q, k, v) = make(rkv, 4, 2, 1, torch.bfloat16, 3)
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    t = rkv.RopeTable(64)
    t.rot_dim = 40
    with pytest.raises(rkv.RkvError):
        ctx.rope(x, pos, t, q[:4], k[:4], v[:4])
    t.rot_dim, t.layout = 64, 2
    with pytest.raises(rkv.RkvError):
        ctx.rope(x, pos, t, q[:4], k[:4], v[:4])
    t.layout = 0
    odd = torch.empty(4 * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(4, 1, 128)
    with pytest.raises(rkv.RkvError):
        ctx.rope(x, pos, t, q[:4], odd, v[:4])
