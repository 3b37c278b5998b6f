"""The 8-bit full cache on the GPU against the fp64 oracle.

Tolerances
  store, rebuild   bit exact (scales are powers of two, every step but the one rounding is exact)
  out              |got - want| <= 2^-8 |want| + 2^-10 S + 1e-30,  S = sum_j p_j |v_j|: half a bf16 step for the output;
                   2^-11 S for the halves that carry p (half an f16 step each), as much again for fp32 logits, exp and sums
  scores           relative 1e-4 + absolute 1e-9 (fp32 logits of magnitude < 100: 100 * 2^-22 = 2.4e-5 relative in p)
  top-K            the oracle's set outside the 1e-5 relative band around the K-th score
"""
import math

import numpy as np
import pytest
import torch

from oracle import quant_oracle as QO
from oracle import rkv_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2411_05787_b200 import rkv, runner, synth
    return rkv, runner, synth


def f64(t):
    return t.detach().double().cpu().numpy()


def codes_of(t):
    return t.detach().cpu().view(torch.uint8).numpy().copy()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def context(rkv, n_seq, n_q, n_kv, max_len, max_small=64, **kw):
    return rkv.Context(n_seq, n_q, n_kv, max_len, max_small, **kw)


def head_rows(c, b, g):
    off, cap = int(c.row_offset[b]), int(c.cap[b])
    return off + g * cap, cap


class Host:
    """A cache's codes and scales as the oracle keeps them."""

    def __init__(self, c, n_kv):
        self.c, self.n_kv = c, n_kv
        self.codes = {"k": codes_of(c.k), "v": codes_of(c.v)}
        self.scale = {"k": f64(c.k_scale), "v": f64(c.v_scale)}
        self.len = c.len.tolist()

    def store(self, k_new, v_new, start=None, count=None):
        for b in range(len(self.len)):
            s = self.len[b] if start is None else start[b]
            n = k_new.shape[1] if count is None else max(count[b], 0)
            for which, x in (("k", k_new), ("v", v_new)):
                for g in range(self.n_kv):
                    r, cap = head_rows(self.c, b, g)
                    QO.store(self.codes[which][r: r + cap], self.scale[which][r // 64: (r + cap) // 64], f64(x[b, :, g]), s, n)
            self.len[b] = min(s + n, cap)

    def check(self):
        for which in "kv":
            assert np.array_equal(self.codes[which], codes_of(getattr(self.c, which))), which
            assert np.array_equal(self.scale[which], f64(getattr(self.c, which + "_scale")), equal_nan=True), which
        assert self.len == self.c.len.tolist()

    def values(self, which, b, g, n):
        r, cap = head_rows(self.c, b, g)
        return QO.values(self.codes[which][r: r + n], self.scale[which][r // 64: (r + cap) // 64])


def filled(synth, lens, n_kv, seed, caps=None, past=0x7f):
    """A cache of random rows of the given lengths; codes past them are NaN, scales of blocks past them too."""
    g = gen(seed)
    c = synth.alloc_quant_cache(caps or [n + 1 for n in lens], n_kv, torch.device("cuda"))
    for which in "kv":
        x = normal(g, c.n_rows, 128)
        codes = getattr(c, which).view(torch.uint8)
        scale = torch.exp2(torch.randint(-8, -3, (c.n_rows // 64,), generator=g, device="cuda").float())
        codes.copy_((x / scale.repeat_interleave(64)[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
        for b, n in enumerate(lens):
            for h in range(n_kv):
                r, cap = head_rows(c, b, h)
                codes[r + n: r + cap] = past
                scale[(r + (n + 63) // 64 * 64) // 64: (r + cap) // 64] = float("nan")
        getattr(c, which + "_scale").copy_(scale)
    c.len.copy_(i32(lens))
    return c


def struct(rkv, c):
    return rkv.quant_cache_struct(c.k, c.v, c.k_scale, c.v_scale, c.row_offset, c.cap, c.len)


# ---------------------------------------------------------------------------------------------------------------- store
@pytest.mark.parametrize("tokens", [1, 2, 63, 64, 65, 129, 700])
@pytest.mark.parametrize("n_kv", [1, 3, 8])
def test_store_appends_bit_exact(mods, tokens, n_kv):
    rkv, runner, synth = mods
    g = gen(tokens * 10 + n_kv)
    lens = [0, 1, 64, 37]
    c = synth.alloc_quant_cache([n + 2 * tokens for n in lens], n_kv, torch.device("cuda"))
    ctx = context(rkv, 4, n_kv, n_kv, 64)
    cs = struct(rkv, c)
    host = Host(c, n_kv)
    first = normal(g, 4, 64, n_kv, 128).to(torch.bfloat16)
    ctx.quant_store(first, first, cs, count=i32(lens))
    host.store(first, first, count=lens)
    host.check()
    for growth in (1.0, 8.0):       # the second rows raise the scale of the block they join
        k = (normal(g, 4, tokens, n_kv, 128) * growth).to(torch.bfloat16)
        v = (normal(g, 4, tokens, n_kv, 128) / growth).to(torch.bfloat16)
        ctx.quant_store(k, v, cs)
        host.store(k, v)
        host.check()
    assert ctx.device_status() == 0


def test_store_start_count_strides_and_rows_it_must_leave(mods):
    rkv, runner, synth = mods
    g = gen(3)
    n_kv, T = 2, 150
    lens = [200, 130, 64, 0, 77]
    c = filled(synth, lens, n_kv, 5, caps=[512] * 5, past=0x55)
    host = Host(c, n_kv)
    wide = normal(g, 5, T, 7, 128).to(torch.bfloat16)       # rows inside a wider projection
    k, v = wide[:, :, 1:3], wide[:, :, 5:7]
    start, count = [200, 100, 63, 0, 10], [150, 3, 0, 65, -4]
    ctx = context(rkv, 5, 4, n_kv, 512)
    ctx.quant_store(k, v, struct(rkv, c), start=i32(start), count=i32(count))
    host.store(k, v, start, count)
    host.check()                    # codes of every other row included; a sequence without new rows is cut to start
    assert c.len.tolist() == [350, 103, 63, 65, 10]
    assert ctx.device_status() == 0


@pytest.mark.parametrize("values", ["zeros", "tiny", "huge", "subnormal", "edge"])
def test_store_extreme_values(mods, values):
    rkv, runner, synth = mods
    g = gen(11)
    x = normal(g, 1, 130, 1, 128)
    if values == "zeros":
        x = x * 0
    elif values == "tiny":
        x = x * 2.0 ** -130
    elif values == "subnormal":
        x[:, :, :, :] = 2.0 ** -133
    elif values == "huge":
        x = x.clamp(-1, 1) * 3e38
    else:                           # 448 times a power of two needs exactly that power, the next bf16 value the next
        x = x.clamp(-1, 1)
        x[0, 0, 0, 0], x[0, 64, 0, 0], x[0, 129, 0, 5] = 1.75, 1.7578125, -1.75
    x = x.to(torch.bfloat16)
    c = synth.alloc_quant_cache([256], 1, torch.device("cuda"))
    host = Host(c, 1)
    ctx = context(rkv, 1, 1, 1, 256)
    ctx.quant_store(x, -x, struct(rkv, c))
    host.store(x, -x)
    host.check()
    ctx.quant_store(x[:, :1] * 0 + 1, x[:, :1] * 0 + 3e38, struct(rkv, c))    # joins the last block
    host.store(x[:, :1] * 0 + 1, x[:, :1] * 0 + 3e38)
    host.check()
    assert ctx.device_status() == 0


def test_store_flags(mods):
    """What only the device can see: rows past the capacity, a start past the length, sizes that do not suit blocks,
    values that are not finite."""
    rkv, runner, synth = mods
    g = gen(12)
    c = filled(synth, [100, 100, 100, 100], 1, 7, caps=[128] * 4)
    x = normal(g, 4, 40, 1, 128).to(torch.bfloat16)
    ctx = context(rkv, 4, 1, 1, 128)
    host = Host(c, 1)
    ctx.quant_store(x, x, struct(rkv, c), start=i32([100, 101, -1, 128]))
    assert ctx.device_status() == rkv.DEV_APPEND_OVERFLOW | rkv.DEV_LEN_CLAMPED
    host.store(x, x, start=[100, 100, 100, 100], count=[40, 0, 0, 0])
    host.check()                                        # 28 of 40 rows fitted; the other three stayed as they were
    assert c.len.tolist() == [128, 100, 100, 100]
    c.cap[1] = 100
    c.row_offset[2] = 300
    c.row_offset[3] = 1 << 20
    ctx.quant_store(x, x, struct(rkv, c), start=i32([128, 0, 0, 0]))
    assert ctx.device_status() == rkv.DEV_APPEND_OVERFLOW | rkv.DEV_BAD_LAYOUT
    assert c.len.tolist() == [128, 100, 100, 100]
    for which in "kv":
        assert np.array_equal(host.codes[which], codes_of(getattr(c, which)))
    x[0, 3, 0, 7], x[0, 5, 0, 1], x[0, 4, 0, 0] = math.inf, -math.inf, math.nan
    c2 = synth.alloc_quant_cache([64], 1, torch.device("cuda"))
    ctx1 = context(rkv, 1, 1, 1, 64)
    h2 = Host(c2, 1)
    ctx1.quant_store(x[:1], x[:1].nan_to_num(0, 0, 0), struct(rkv, c2))
    h2.store(x[:1], x[:1].nan_to_num(0, 0, 0))
    h2.check()
    assert ctx1.device_status() == rkv.DEV_NONFINITE


# ------------------------------------------------------------------------------------------------------------ attention
def reference(host, q, n_kv, lens, scale=None):
    """Per sequence: out [Hq, 128], S [Hq, 128] = sum p |v|, p [Hq, n]; None for an empty one."""
    ref = []
    for b, n in enumerate(lens):
        if n == 0:
            ref.append(None)
            continue
        k = np.stack([host.values("k", b, g, n) for g in range(n_kv)])
        v = np.stack([host.values("v", b, g, n) for g in range(n_kv)])
        out, p, _ = O.decode_attention(f64(q[b]), k, v, scale)
        mass, _, _ = O.decode_attention(f64(q[b]), k, np.abs(v), scale)
        ref.append((out, mass, p))
    return ref


def check_out(got, ref, what=""):
    out, mass, _ = ref
    err = np.abs(f64(got) - out)
    tol = 2.0 ** -8 * np.abs(out) + 2.0 ** -10 * mass + 1e-30
    assert (err <= tol).all(), f"{what}: {np.max(err / tol):.2f} tolerances"


def check_scores(got, p, group, what=""):
    want = p.reshape(-1, group, p.shape[1]).max(axis=1)
    err = np.abs(f64(got)[:, : p.shape[1]] - want)
    assert (err <= 1e-4 * want + 1e-9).all(), what


@pytest.mark.parametrize("group", [1, 3, 4, 7, 8])
@pytest.mark.parametrize("lens", [[1], [63], [64, 65], [127, 128, 129, 0], [1000], [4097, 1, 300], [20000, 8191]])
def test_attention_and_scores(mods, lens, group):
    rkv, runner, synth = mods
    n_kv = 2
    c = filled(synth, lens, n_kv, group * 100 + len(lens))
    g = gen(group)
    q = (normal(g, len(lens), n_kv * group, 128) * 1.5).to(torch.bfloat16)
    ctx = context(rkv, len(lens), n_kv * group, n_kv, max(lens) + 64)
    out = torch.full_like(q, 7.0)
    scores = torch.full((len(lens), n_kv, max(lens)), -1.0, device="cuda")
    cs = struct(rkv, c)
    ctx.quant_full_attention(q, cs, out, max_len_hint=max(lens))
    ctx.score_keys(q, cs, i32([1] * len(lens)), 1, scores=scores)
    alone = torch.full_like(q, 7.0)
    ctx.quant_full_attention(q, cs, alone, max_len_hint=max(lens), keep_logits=False)
    assert torch.equal(out, alone)
    ref = reference(Host(c, n_kv), q, n_kv, lens)
    for b, n in enumerate(lens):
        if n == 0:
            assert (out[b] == 0).all() and (scores[b] == -1).all()
            continue
        check_out(out[b], ref[b], f"sequence {b}")
        check_scores(scores[b], ref[b][2], group, f"sequence {b}")
        assert (scores[b, :, n:] == -1).all()
    assert ctx.device_status() == 0


@pytest.mark.parametrize("n_seq,n_kv,group,most", [(2, 1, 4, 40000), (3, 2, 7, 2500), (3, 2, 7, 9000), (40, 3, 2, 1500),
                                                   (40, 3, 2, 2500), (256, 1, 8, 1100), (257, 1, 1, 1100), (300, 2, 4, 900)])
def test_attention_ragged_batches(mods, n_seq, n_kv, group, most):
    """Batches whose heads share CTAs: lengths from nothing to the longest, masked sequences, runs that end inside heads,
    one head with more tiles than it may leave partials, and more sequences than the balanced form takes."""
    rkv, runner, synth = mods
    rng = np.random.default_rng(n_seq)
    lens = [most] + [int(x) for x in np.exp(rng.uniform(0, np.log(most), n_seq - 1))]
    for i in range(3, n_seq, 7):
        lens[i] = 0
    c = filled(synth, lens, n_kv, n_seq)
    q = normal(gen(n_seq), n_seq, n_kv * group, 128).to(torch.bfloat16)
    on = [0 if i % 5 == 4 else 1 for i in range(n_seq)]
    ctx = context(rkv, n_seq, n_kv * group, n_kv, most)
    cs = struct(rkv, c)
    ref = reference(Host(c, n_kv), q, n_kv, lens)
    for active, hint in ((None, 0), (i32(on), most)):
        out = torch.full_like(q, 7.0)
        scores = torch.full((n_seq, n_kv, most), -1.0, device="cuda")
        ctx.quant_full_attention(q, cs, out, active=active, max_len_hint=hint)
        ctx.score_keys(q, cs, i32([1] * n_seq), 1, active=active, scores=scores)
        alone = torch.full_like(q, 7.0)
        ctx.quant_full_attention(q, cs, alone, active=active, max_len_hint=hint, keep_logits=False)
        assert torch.equal(out, alone)
        for b, n in enumerate(lens):
            if active is not None and not on[b]:
                assert (out[b] == 7).all() and (scores[b] == -1).all()
            elif n == 0:
                assert (out[b] == 0).all()
            else:
                check_out(out[b], ref[b], f"sequence {b}")
                check_scores(scores[b], ref[b][2], group, f"sequence {b}")
                assert (scores[b, :, n:] == -1).all()
    out = torch.full_like(q, 7.0)
    ctx.quant_full_attention(q, cs, out, active=i32([0] * n_seq))
    assert (out == 7).all() and ctx.device_status() == 0


def test_attention_masked_batch_leaves_the_others(mods):
    rkv, runner, synth = mods
    lens, n_kv, group = [500, 900, 0, 64, 2000], 2, 4
    c = filled(synth, lens, n_kv, 21)
    q = normal(gen(1), 5, 8, 128).to(torch.bfloat16)
    ctx = context(rkv, 5, 8, n_kv, 2048)
    out = torch.full_like(q, 7.0)
    scores = torch.full((5, n_kv, 2000), -1.0, device="cuda")
    active = i32([1, 0, 1, 0, 1])
    cs = struct(rkv, c)
    ctx.quant_full_attention(q, cs, out, active=active, max_len_hint=2000)
    ctx.score_keys(q, cs, i32([1] * 5), 1, active=active, scores=scores)
    ref = reference(Host(c, n_kv), q, n_kv, lens)
    for b in (1, 3):
        assert (out[b] == 7).all() and (scores[b] == -1).all()
    assert (out[2] == 0).all()
    for b in (0, 4):
        check_out(out[b], ref[b])
        check_scores(scores[b], ref[b][2], group)
    ctx.quant_full_attention(q, cs, out, active=i32([0] * 5))
    for b in (0, 4):
        check_out(out[b], ref[b])
    assert ctx.device_status() == 0


@pytest.mark.parametrize("what", ["scales", "peaked", "tail", "large q", "small q", "zero q", "any scale", "softmax scale"])
def test_attention_extremes(mods, what):
    """Where the halves could run out of range: blocks of very different scale, one position that holds all the weight
    beside a long tail that together matters, queries of extreme magnitude, scales that are no powers of two."""
    rkv, runner, synth = mods
    n, n_kv, group = 3000, 2, 4
    c = filled(synth, [n], n_kv, 31)
    g = gen(32)
    q = normal(g, 1, 8, 128)
    kw = {}
    if what == "scales":
        c.v_scale.mul_(torch.exp2(torch.randint(-60, 60, c.v_scale.shape, generator=g, device="cuda").float()))
        c.v_scale.view(n_kv, -1)[:, 3] = 0.0
    elif what == "any scale":
        c.v_scale.mul_(torch.rand(c.v_scale.shape, generator=g, device="cuda") + 0.5)
        c.k_scale.mul_(torch.rand(c.k_scale.shape, generator=g, device="cuda") + 0.5)
    elif what in ("peaked", "tail"):
        q = torch.zeros_like(q)
        q[..., 0] = 1.0
        k = c.k.view(torch.uint8)
        for h in range(n_kv):
            r, cap = head_rows(c, 0, h)
            k[r: r + n] = 0
            c.k_scale[r // 64: (r + cap) // 64] = 1.0
            k[r + 1700, 0] = int(QO.encode(np.array([88.0 if what == "tail" else 448.0]))[0])
        c.v.view(torch.uint8).bitwise_and_(0x7f)        # positive values: the tail's weight shows
        if what == "tail":                              # 8 nats: 3000 e^-8 = 1.0 of the heavy position's weight
            q *= 1.03
    elif what == "large q":
        q *= 2.0 ** 100
        c.k_scale.mul_(2.0 ** -100)
    elif what == "small q":
        q *= 2.0 ** -120
        c.k_scale.mul_(2.0 ** 100).mul_(2.0 ** 20)
    elif what == "zero q":
        q[:, 1] = 0
    else:
        kw = dict(softmax_scale=0.3)
    q = q.to(torch.bfloat16)
    ctx = context(rkv, 1, 8, n_kv, n, **kw)
    out = torch.empty((1, 8, 128), dtype=torch.bfloat16, device="cuda")
    scores = torch.zeros((1, n_kv, n), device="cuda")
    cs = struct(rkv, c)
    ctx.quant_full_attention(q, cs, out)
    ctx.score_keys(q, cs, i32([1]), 1, scores=scores)
    ref = reference(Host(c, n_kv), q, n_kv, [n], kw.get("softmax_scale"))
    check_out(out[0], ref[0], what)
    check_scores(scores[0], ref[0][2], group, what)
    assert ctx.device_status() == 0


@pytest.mark.parametrize("lens", [[700], [6000], [700, 350], [9000, 64, 4000]])
@pytest.mark.parametrize("where", ["first", "last", "every other"])
def test_attention_large_values_of_no_weight(mods, lens, where):
    """Blocks whose values are 2^70 times as large as the others' and whose logits lie 100 nats below: they weigh nothing
    (e^-100 2^70 = 2^-74), and must not cost the others their bits, wherever they stand."""
    rkv, runner, synth = mods
    n_kv, group = 2, 4
    c = filled(synth, lens, n_kv, 61)
    q = torch.zeros((len(lens), n_kv * group, 128), device="cuda")
    q[..., 0], q[..., 1:] = 8.0, normal(gen(62), len(lens), n_kv * group, 127) * 0.2
    q = q.to(torch.bfloat16)
    k = c.k.view(torch.uint8)
    low = int(QO.encode(np.array([-144.0]))[0])
    for b, n in enumerate(lens):
        blocks = (n + 63) // 64
        for h in range(n_kv):
            r, cap = head_rows(c, b, h)
            k[r: r + n, 0] = 0
            c.k_scale[r // 64: r // 64 + blocks] = 1.0
            k[r: r + n, 1:] = 0x30                                     # 0.5: every other logit alike
            for i in range(blocks):
                if blocks > 1 and (i < 2 if where == "first" else i >= blocks - 2 if where == "last" else i % 2 == 0) and i != 1:
                    k[r + 64 * i: r + min(64 * i + 64, n), 0] = low    # 8 * -144 / sqrt(128) = -101.8
                    c.v_scale[r // 64 + i] *= 2.0 ** 70
    ctx = context(rkv, len(lens), n_kv * group, n_kv, max(lens))
    out = torch.empty_like(q)
    ctx.quant_full_attention(q, struct(rkv, c), out)
    ref = reference(Host(c, n_kv), q, n_kv, lens)
    for b in range(len(lens)):
        check_out(out[b], ref[b], f"sequence {b}")
    assert ctx.device_status() == 0


@pytest.mark.parametrize("max_len", [512, 16384])
def test_attention_flags(mods, max_len):
    """(The bound decides the form: clusters, or runs balanced over the batch.)"""
    rkv, runner, synth = mods
    lens = [300, 300, 300]
    c = filled(synth, lens, 1, 41, caps=[320] * 3)
    q = normal(gen(1), 3, 4, 128).to(torch.bfloat16)
    ctx = context(rkv, 3, 4, 1, max_len)
    out = torch.full_like(q, 7.0)
    ref = reference(Host(c, 1), q, 1, lens)
    c.row_offset[1] += 32
    ctx.quant_full_attention(q, struct(rkv, c), out)
    assert ctx.device_status() == rkv.DEV_BAD_LAYOUT
    assert (out[1] == 0).all()
    check_out(out[0], ref[0])
    check_out(out[2], ref[2])
    c.row_offset[1] -= 32
    ref256 = reference(Host(c, 1), q, 1, [256] * 3)
    ctx.quant_full_attention(q, struct(rkv, c), out, max_len_hint=256)        # longer than the bound: clamped
    assert ctx.device_status() == rkv.DEV_LEN_CLAMPED
    for b in range(3):
        check_out(out[b], ref256[b])
    c.k.view(torch.uint8)[5] = 0x7f                                            # a NaN row inside the length
    scores = torch.zeros((3, 1, 320), device="cuda")
    cs = struct(rkv, c)
    ctx.quant_full_attention(q, cs, out, max_len_hint=320)
    ctx.score_keys(q, cs, i32([1] * 3), 1, scores=scores)
    assert ctx.device_status() & rkv.DEV_NONFINITE


def test_smallest_cache(mods):
    """One block in all: 64 rows, fewer than a tile of the pass."""
    rkv, runner, synth = mods
    for n in (1, 64):
        c = filled(synth, [n], 1, n, caps=[64])
        q = normal(gen(n), 1, 1, 128).to(torch.bfloat16)
        ctx = context(rkv, 1, 1, 1, 64)
        out = torch.empty_like(q)
        ctx.quant_full_attention(q, struct(rkv, c), out)
        check_out(out[0], reference(Host(c, 1), q, 1, [n])[0])
        assert ctx.device_status() == 0


def test_attention_right_behind_a_store(mods):
    """Store and attention back to back many times: the pass must not read its first tiles before the store is done
    (and may behind other launches)."""
    rkv, runner, synth = mods
    n_kv, n = 2, 300
    c = synth.alloc_quant_cache([n + 40], n_kv, torch.device("cuda"))
    ctx = context(rkv, 1, 8, n_kv, n + 64)
    cs = struct(rkv, c)
    g = gen(9)
    host = Host(c, n_kv)
    x = normal(g, 1, n, n_kv, 128).to(torch.bfloat16)
    ctx.quant_store(x, x, cs)
    host.store(x, x)
    qs, outs, news = [], [], []
    for i in range(20):
        q, k = normal(g, 1, 8, 128).to(torch.bfloat16), (normal(g, 1, 1, n_kv, 128) * 3).to(torch.bfloat16)
        qs.append(q); news.append(k); outs.append((torch.empty_like(q), torch.empty_like(q)))
    torch.cuda.synchronize()
    for q, k, (a, b) in zip(qs, news, outs):
        ctx.quant_store(k, k, cs)
        ctx.quant_full_attention(q, cs, a)
        ctx.quant_full_attention(q, cs, b)
    for q, k, (a, b) in zip(qs, news, outs):
        host.store(k, k)
        ref = reference(host, q, n_kv, host.len)
        check_out(a[0], ref[0])
        assert torch.equal(a, b)
    host.check()
    assert ctx.device_status() == 0


def test_selection_after_scores_without_one(mods):
    """A captured graph of attention and scores alone, replayed between full steps, leaves the full steps' selections
    as they are (the keys' histogram starts from zero in every pass)."""
    rkv, runner, synth = mods
    c = filled(synth, [5000], 2, 3)
    q = normal(gen(3), 1, 8, 128).to(torch.bfloat16)
    ctx = context(rkv, 1, 8, 2, 5120, 300)
    cs = struct(rkv, c)
    out, idx = torch.empty_like(q), torch.empty((1, 2, 300), dtype=torch.int32, device="cuda")
    scores = torch.zeros((1, 2, 5120), device="cuda")
    k_small = i32([300])
    ctx.quant_full_step(q, cs, k_small, 300, out, idx)
    want = idx.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            ctx.quant_full_attention(q, cs, out)
            ctx.score_keys(q, cs, k_small, 300, scores=scores)
        for _ in range(3):
            graph.replay()
            idx.fill_(-7)
            ctx.quant_full_step(q, cs, k_small, 300, out, idx)
            assert torch.equal(idx, want)
    assert ctx.device_status(side) == 0


@pytest.mark.parametrize("halves", [False, True])
def test_captured_quant_step_leaves_the_bf16_selection_alone(mods, halves):
    """One context for a bf16 and an 8-bit cache: scores without a selection leave keys in the histogram; a full step over
    the 8-bit cache that is only captured has not cleared them, and the bf16 full step behind it must."""
    rkv, runner, synth = mods
    n = 3000
    c = filled(synth, [n], 2, 3)
    bf = synth.alloc_cache([n], [n], 2, torch.device("cuda"))
    g = gen(5)
    bf.k.copy_(normal(g, *bf.k.shape)); bf.v.copy_(normal(g, *bf.v.shape))
    bs = rkv.cache_struct(bf.k, bf.v, bf.row_offset, bf.cap, bf.len)
    cs = struct(rkv, c)
    q = normal(g, 1, 8, 128).to(torch.bfloat16)
    ctx = context(rkv, 1, 8, 2, 3200, 256)
    out, k_small = torch.empty_like(q), i32([256])
    idx, want = (torch.empty((1, 2, 256), dtype=torch.int32, device="cuda") for _ in range(2))
    ctx.full_step(q, bs, k_small, 256, out, want)
    ctx.full_attention(q, bs, out)
    ctx.score_keys(q, bs, k_small, 256)                 # keys counted, nothing selected
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            if halves:
                ctx.quant_full_attention(q, cs, out)
                ctx.score_keys(q, cs, k_small, 256)
                ctx.select_topk(None, cs, k_small, 256, idx)
            else:
                ctx.quant_full_step(q, cs, k_small, 256, out, idx)
        idx.fill_(-7)
        ctx.full_step(q, bs, k_small, 256, out, idx)
        assert torch.equal(idx, want)
        graph.replay()
        ctx.full_step(q, bs, k_small, 256, out, idx)
        assert torch.equal(idx, want)
    assert ctx.device_status(side) == 0


# -------------------------------------------------------------------------------------------------------------- rebuild
@pytest.mark.parametrize("keep", [1, 63, 64, 65, 200, 1000])
def test_rebuild_bit_exact(mods, keep):
    rkv, runner, synth = mods
    lens, n_kv = [1000, 64, 1, 0, 500], 3
    c = filled(synth, lens, n_kv, keep)
    host = Host(c, n_kv)
    rng = np.random.default_rng(keep)
    ks = [min(keep, 1000), min(keep, 64), keep, keep, max(keep // 2, 1)]
    idx = np.full((5, n_kv, keep), -1, np.int32)
    for b, n in enumerate(lens):
        m = min(ks[b], n)
        for g in range(n_kv):
            idx[b, g, :m] = np.sort(rng.permutation(n)[:m])
    small = synth.alloc_cache([keep + 3] * 5, [9] * 5, n_kv, torch.device("cuda"), fill=5.0)
    ctx = context(rkv, 5, n_kv, n_kv, 1024, keep)
    sc = rkv.cache_struct(small.k, small.v, small.row_offset, small.cap, small.len)
    ctx.quant_gather_small(torch.from_numpy(idx).cuda(), i32(ks), keep, struct(rkv, c), sc, active=i32([1, 1, 1, 1, 0]))
    want = {w: np.full((5 * n_kv * (keep + 3), 128), 5.0) for w in "kv"}
    for b in range(4):
        m = min(ks[b], lens[b])
        for g in range(n_kv):
            r = (b * n_kv + g) * (keep + 3)
            for w in "kv":
                if m:
                    want[w][r: r + m] = host.values(w, b, g, lens[b])[idx[b, g, :m]]
    for w in "kv":
        assert np.array_equal(want[w], f64(getattr(small, w))), w      # rows behind each rebuilt cache included
    assert small.len.tolist() == [min(ks[b], lens[b]) for b in range(4)] + [9]
    assert ctx.device_status() == 0


def test_rebuild_flags_and_any_scale(mods):
    rkv, runner, synth = mods
    c = filled(synth, [200], 1, 3)
    c.k_scale.mul_(1.37)
    small = synth.alloc_cache([8], [0], 1, torch.device("cuda"), fill=5.0)
    ctx = context(rkv, 1, 1, 1, 256, 8)
    sc = rkv.cache_struct(small.k, small.v, small.row_offset, small.cap, small.len)
    idx = i32([[[0, 199, 200, 1 << 30, -7, -1, 63, 64]]])
    ctx.quant_gather_small(idx, i32([8]), 8, struct(rkv, c), sc)
    assert ctx.device_status() == rkv.DEV_BAD_INDEX
    host = Host(c, 1)
    for r, j in ((0, 0), (1, 199), (6, 63), (7, 64)):
        want = torch.from_numpy(host.values("k", 0, 0, 200)[j]).float().to(torch.bfloat16)
        assert torch.equal(small.k[r].cpu(), want)
    assert (small.k[2:6] == 5).all()
    small.cap[0] = 2                       # fewer rows than selected: cut and flagged
    small.k.fill_(5.0)
    ctx.quant_gather_small(i32([[[0, 1, 2, 3, 4, 5, 6, 7]]]), i32([8]), 8, struct(rkv, c), sc)
    assert ctx.device_status() == rkv.DEV_LEN_CLAMPED
    assert small.len.tolist() == [2] and (small.k[2:] == 5).all() and not (small.k[:2] == 5).all()
    c.len[0] = 300                         # longer than the cache: cut and flagged
    ctx.quant_gather_small(i32([[[199, 255, 256, 299, -1, -1, -1, -1]]]), i32([2]), 8, struct(rkv, c), sc)
    assert ctx.device_status() == rkv.DEV_LEN_CLAMPED
    c.len[0] = 200
    c.cap[0] = 250
    ctx.quant_gather_small(idx, i32([8]), 8, struct(rkv, c), sc)
    assert ctx.device_status() == rkv.DEV_BAD_LAYOUT


# ------------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("shape", [(4, 8, [2500]), (7, 2, [1500, 70, 3000])])
def test_prompt_full_step_rebuild_and_partial_steps(mods, shape):
    """A prompt joins the 8-bit cache, a full step selects, the small cache is rebuilt from it, tokens are appended to
    both, and a full step follows: each call against the oracle on the oracle's own cache."""
    rkv, runner, synth = mods
    group, n_kv, lens = shape
    n_q, B, T = group * n_kv, len(lens), max(lens)
    g = gen(sum(lens))
    ks = [min(200, n) for n in lens]
    cache = synth.alloc_quant_cache([n + 8 for n in lens], n_kv, torch.device("cuda"))
    ctx = context(rkv, B, n_q, n_kv, int(cache.cap.max()), 256)
    st = runner.QuantLayerState(ctx, cache, ks, 8, n_q, n_kv, want_scores=True)
    host = Host(cache, n_kv)
    k, v = normal(g, B, T, n_kv, 128).to(torch.bfloat16), normal(g, B, T, n_kv, 128).to(torch.bfloat16)
    st.store_prompt(k, v, count=i32(lens))
    host.store(k, v, count=lens)
    host.check()

    def full(q, halves):
        if halves:
            out = st.refresh_attention(q).clone()
            st.refresh_select(q)
        else:
            out = st.refresh(q).clone()
        idx = st.topk_idx.cpu().numpy()
        ref = reference(host, q, n_kv, host.len)
        kept = {}
        for b in range(B):
            check_out(out[b], ref[b], f"full {b}")
            check_scores(st.scores[b], ref[b][2], group)
            want = ref[b][2].reshape(n_kv, group, -1).max(axis=1)
            for h in range(n_kv):
                why = O.check_topk_set(want[h], ks[b], idx[b, h, : ks[b]])
                assert why is None, why
                kept[b, h] = idx[b, h, : ks[b]]
        assert torch.equal(st.q_last_full, q)
        return kept

    def small_check(q, kept, extra, out):
        for b in range(B):
            kk = np.stack([np.concatenate([host.values("k", b, h, host.len[b])[kept[b, h]], extra[0][b][h]]) for h in range(n_kv)])
            vv = np.stack([np.concatenate([host.values("v", b, h, host.len[b])[kept[b, h]], extra[1][b][h]]) for h in range(n_kv)])
            want, _, _ = O.decode_attention(f64(q[b]), kk, vv)
            mass, _, _ = O.decode_attention(f64(q[b]), kk, np.abs(vv))
            # the bf16 small cache's attention carries p as bf16: 2^-8 of S, and fp32 noise
            assert (np.abs(f64(out[b]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * mass).all()

    for halves in (False, True):
        kept = full(normal(g, B, n_q, 128).to(torch.bfloat16), halves)
        extra = ([[np.zeros((0, 128))] * n_kv for _ in range(B)], [[np.zeros((0, 128))] * n_kv for _ in range(B)])
        for step in range(3):
            q = normal(g, B, n_q, 128).to(torch.bfloat16)
            kn, vn = (normal(g, B, n_kv, 128) * 2).to(torch.bfloat16), normal(g, B, n_kv, 128).to(torch.bfloat16)
            out = st.append_partial(q, kn, vn)
            host.store(kn[:, None], vn[:, None])
            host.check()
            for e, x in zip(extra, (kn, vn)):
                for b in range(B):
                    e[b] = [np.concatenate([e[b][h], f64(x[b, h])[None]]) for h in range(n_kv)]
            small_check(q, kept, extra, out)
    assert ctx.device_status() == 0


def test_schedules_take_quant_layers(mods):
    """DeferredRefresh and OverlappedRefresh over 8-bit layers give what the calls in order give."""
    rkv, runner, synth = mods
    n_q, n_kv, n = 8, 2, 1200

    def layers(share):
        g = gen(77)
        ctxs = [context(rkv, 1, n_q, n_kv, n + 64, 160) for _ in range(share)]
        made = []
        for l in range(4):
            cache = synth.alloc_quant_cache([n + 8], n_kv, torch.device("cuda"))
            st = runner.QuantLayerState(ctxs[l % share], cache, [128], 8, n_q, n_kv)
            x = normal(g, 1, n, n_kv, 128).to(torch.bfloat16)
            st.store_prompt(x, x)
            made.append(st)
        return made

    g = gen(78)
    q = normal(g, 4, 1, n_q, 128).to(torch.bfloat16)
    k, v = normal(g, 4, 1, n_kv, 128).to(torch.bfloat16), normal(g, 4, 1, n_kv, 128).to(torch.bfloat16)
    plain = layers(1)
    for l, st in enumerate(plain):
        st.append(k[l], v[l])
        st.refresh(q[l])
    early = lambda ls: runner.DeferredRefresh(ls, early_scores=True)
    for make, share in ((runner.DeferredRefresh, 4), (early, 4), (runner.OverlappedRefresh, 2)):
        ls = layers(share)
        torch.cuda.synchronize()
        make(ls).run(lambda l: q[l], lambda l: k[l], lambda l: v[l])
        torch.cuda.synchronize()
        for a, b in zip(plain, ls):
            assert torch.equal(a.topk_idx, b.topk_idx) and torch.equal(a.small.k[: 128], b.small.k[: 128])
            assert (a.out.float() - b.out.float()).abs().max() <= 2.0 ** -8 * a.out.float().abs().max()   # (the fold's order)
            assert b.ctx.device_status() == 0


def test_checked_tokens_over_quant_layers(mods):
    """The dynamic schedule's check token over a ragged batch: some sequences refresh, the others take the partial step,
    under device masks, as the calls in order do."""
    rkv, runner, synth = mods
    n_q, n_kv, lens, layers = 8, 2, [900, 300, 1200], 3

    def build(share):
        g = gen(91)
        ctxs = [context(rkv, 3, n_q, n_kv, 1280, 160) for _ in range(share)]
        made = []
        for l in range(layers):
            st = runner.QuantLayerState(ctxs[l % share], synth.alloc_quant_cache([n + 8 for n in lens], n_kv, torch.device("cuda")),
                                        [128, 64, 128], 8, n_q, n_kv)
            x = normal(g, 3, max(lens), n_kv, 128).to(torch.bfloat16)
            st.store_prompt(x, x, count=i32(lens))
            st.refresh(normal(g, 3, n_q, 128).to(torch.bfloat16))
            made.append(st)
        return made

    g = gen(92)
    k, v = normal(g, layers, 3, n_kv, 128).to(torch.bfloat16), normal(g, layers, 3, n_kv, 128).to(torch.bfloat16)
    plain = build(1)
    q = torch.stack([st.q_last_full for st in plain])
    q[:, 1] = normal(g, layers, n_q, 128).to(torch.bfloat16)            # the second sequence's query has moved on
    for l, st in enumerate(plain):
        st.check_trigger(q[l], 0.9)
        assert st.flag.tolist() == [0, 1, 0]
        st.append_partial(q[l], k[l], v[l], active=st.not_flag)
        st.refresh(q[l], active=st.flag)
    for make, share in ((runner.DeferredRefresh, layers), (runner.OverlappedRefresh, 2)):
        ls = build(share)
        torch.cuda.synchronize()
        make(ls).run_checked(lambda l: q[l], lambda l: k[l], lambda l: v[l], 0.9)
        torch.cuda.synchronize()
        for a, b in zip(plain, ls):
            assert b.full.len.tolist() == [n + 1 for n in lens] and torch.equal(a.small.len, b.small.len)
            assert torch.equal(a.topk_idx, b.topk_idx) and torch.equal(a.small.k, b.small.k) and torch.equal(a.small.v, b.small.v)
            assert torch.equal(a.full.k.view(torch.uint8), b.full.k.view(torch.uint8))
            assert (a.out.float() - b.out.float()).abs().max() <= 2.0 ** -8 * a.out.float().abs().max()
            assert b.ctx.device_status() == 0


def test_captured_and_replayed_on_another_stream(mods):
    """The chain of one token as a graph: replays on a side stream append, attend, select and rebuild as eager calls do."""
    rkv, runner, synth = mods
    n_q, n_kv, n = 8, 2, 700

    def state():
        g = gen(5)
        cache = synth.alloc_quant_cache([n + 16], n_kv, torch.device("cuda"))
        st = runner.QuantLayerState(context(rkv, 1, n_q, n_kv, n + 16, 72), cache, [64], 8, n_q, n_kv)
        x = normal(g, 1, n, n_kv, 128).to(torch.bfloat16)
        st.store_prompt(x, x)
        return st, normal(g, 1, n_q, 128).to(torch.bfloat16), normal(g, 1, n_kv, 128).to(torch.bfloat16)

    def token(st, q, k):
        st.append_refresh_attention(q, k, k)
        st.refresh_select(q)

    eager, q, k = state()
    for _ in range(4):
        token(eager, q, k)
    st, q, k = state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token(st, q, k)                     # once before the capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            token(st, q, k)
        for _ in range(3):
            graph.replay()
    torch.cuda.synchronize()
    assert st.full.len.tolist() == [n + 4]
    assert torch.equal(eager.out, st.out) and torch.equal(eager.topk_idx, st.topk_idx)
    assert torch.equal(eager.full.k.view(torch.uint8), st.full.k.view(torch.uint8))
    assert torch.equal(eager.small.k, st.small.k)
    assert st.ctx.device_status() == 0


def test_select_completes_the_pass_it_belongs_to(mods):
    rkv, runner, synth = mods
    c, d = filled(synth, [300], 2, 1), filled(synth, [300], 2, 2)
    q = normal(gen(1), 1, 8, 128).to(torch.bfloat16)
    ctx = context(rkv, 1, 8, 2, 512, 64)
    out, idx = torch.empty_like(q), torch.empty((1, 2, 64), dtype=torch.int32, device="cuda")
    cs, ds = struct(rkv, c), struct(rkv, d)
    k_small = i32([64])
    with pytest.raises(rkv.RkvError):                   # nothing to complete
        ctx.select_topk(q, cs, k_small, 64, idx)
    ctx.quant_full_attention(q, cs, out, keep_logits=False)
    with pytest.raises(rkv.RkvError):                   # no logits were kept
        ctx.select_topk(q, cs, k_small, 64, idx)
    ctx.quant_full_attention(q, cs, out)
    with pytest.raises(rkv.RkvError):                   # another cache
        ctx.select_topk(q, ds, k_small, 64, idx)
    ctx.select_topk(q, cs, k_small, 64, idx)
    with pytest.raises(rkv.RkvError):
        ctx.quant_full_attention(q, cs, out, max_len_hint=513)
    with pytest.raises(rkv.RkvError):
        ctx.quant_full_step(q, cs, k_small, 65, out, torch.empty((1, 2, 65), dtype=torch.int32, device="cuda"))
    odd = torch.empty(q.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view(q.shape)
    with pytest.raises(rkv.RkvError):                   # not on a 16-byte boundary
        ctx.quant_full_attention(odd, cs, out)
    assert ctx.device_status() == 0
