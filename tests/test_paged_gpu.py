"""The paged cache on the GPU against the fp64 oracle.

Tolerances
  append    queries and keys as rkv_rope's: 2^-8 |want| (half a bf16 step) + 2^-20 amp (|x| + |y|); values 2^-8 |want|, bit
            exact where they come as bf16; bounds are bit exact against the stored keys
  pages     equal to the oracle's (scores in 64 bits on both sides)
  out       |got - want| <= 2^-8 |want| (the output's half bf16 step) + 2^-8 (S + |want|) + 2^-11 S + 1e-30,  S = sum_j p_j |v_j|:
            with p_j rounded to p_j (1 + d_j), |d_j| <= 2^-8, in numerator and denominator alike, the quotient is off by
            |sum p_j d_j (v_j - out)| / sum p_j (1 + d_j), which is at most 2^-8 (S + |out|) to first order; 2^-11 S for fp32
            logits (|s| < 100: 100 * 2^-22), ex2 and sums, and the second order
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
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


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Pool:
    """A pool of pages, some of them handed out to sequences of the given room (positions)."""

    def __init__(self, rkv, rooms, n_kv, page, seed, lens=None, bounds=True, spare=3, shared=0):
        g = gen(seed)
        self.rkv, self.page, self.n_kv = rkv, page, n_kv
        each = [-(-r // page) for r in rooms]
        n = shared + sum(max(e - shared, 0) for e in each) + spare
        order = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
        self.k = normal(g, n, n_kv, page, 128).to(torch.bfloat16)
        self.v = (normal(g, n, n_kv, page, 128) + normal(g, 128)).to(torch.bfloat16)
        self.table = torch.full((len(rooms), max(max(each), 1)), -1, dtype=torch.int32, device="cuda")
        at = shared
        for b, e in enumerate(each):
            mine = max(e - shared, 0)
            self.table[b, : min(shared, e)] = order[: min(shared, e)]
            self.table[b, shared: shared + mine] = order[at: at + mine]
            at += mine
        self.shared = order[:shared].clone() if shared else None
        self.len = i32(list(lens) if lens is not None else [0] * len(rooms))
        self.k_min = self.k_max = None
        if bounds:
            self.k_min, self.k_max = self.k.amin(2), self.k.amax(2)
            for b, n_b in enumerate(lens or []):
                if n_b % page:
                    p = int(self.table[b, n_b // page])
                    self.k_min[p], self.k_max[p] = (f(self.k[p, :, : n_b % page], 1) for f in (torch.amin, torch.amax))

    def struct(self):
        return self.rkv.paged_cache_struct(self.k, self.v, self.table, self.len, self.k_min, self.k_max)

    def host(self, b, n):
        t = self.table[b].tolist()
        return tuple(PO.rows(f64(x), t, self.page, n) for x in (self.k, self.v))


def check_out(got, want, size, why=""):
    got = f64(got)
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * (size + np.abs(want)) + 2.0 ** -11 * size + 1e-30
    assert (np.abs(got - want) <= tol).all(), (why, np.max(np.abs(got - want) / tol))


# --------------------------------------------------------------------------------------------------------------- append
def check_append(rkv, pool, x, start, count, rot, layout, table, q, before, why=""):
    """What an append of x [B, T, heads * 128] at `start` has left, from the state `before` (a dict of clones)."""
    B, T = x.shape[:2]
    n_kv, page = pool.n_kv, pool.page
    nq = x.shape[2] // 128 - 2 * n_kv
    xs = f64(x).reshape(B, T, nq + 2 * n_kv, 128)
    want_k, want_v = (before[m].clone() for m in "kv")
    want_lo, want_hi = (None, None) if pool.k_min is None else (f64(before["k_min"]), f64(before["k_max"]))
    got_k, got_v = f64(pool.k), f64(pool.v)
    touched = torch.zeros(pool.k.shape[:3], dtype=torch.bool)
    for b in range(B):
        n = count[b]
        if n == 0:
            assert (q[b] == 7).all(), why
            continue
        pos = np.arange(start[b], start[b] + n)
        y = xs[b, :n].copy()
        size = np.abs(y)
        amp = 1.0
        if table is not None:
            f, amp = table
            y[:, : nq + n_kv] = QO.rope(y[:, : nq + n_kv], pos, f, amp, layout)
            r = rot // 2
            i = np.arange(r)
            u, w = (i, i + r) if layout == "half" else (2 * i, 2 * i + 1)
            both = np.abs(xs[b, :n][..., u]) + np.abs(xs[b, :n][..., w])
            size[..., u] = size[..., w] = both
        tol = 2.0 ** -8 * np.abs(y) + 2.0 ** -20 * amp * size
        assert (np.abs(f64(q[b, :n]) - y[:, :nq]) <= tol[:, :nq]).all(), why
        assert (q[b, n:] == 7).all(), why                    # rows that nothing was appended for
        for t, p in enumerate(pos):
            pg, r = PO.place(pool.table[b].tolist(), page, int(p))
            touched[pg, :, r] = True
            assert (np.abs(got_k[pg, :, r] - y[t, nq: nq + n_kv]) <= tol[t, nq: nq + n_kv]).all(), why
            assert (np.abs(got_v[pg, :, r] - y[t, nq + n_kv:]) <= 2.0 ** -8 * np.abs(y[t, nq + n_kv:])).all(), why
            if x.dtype == torch.bfloat16:
                assert np.array_equal(got_v[pg, :, r], y[t, nq + n_kv:]), why
        if want_lo is not None:
            for i in range(pos[0] // page, pos[-1] // page + 1):
                pg = int(pool.table[b, i])
                lo, hi = max(pos[0] - i * page, 0), min(pos[-1] + 1 - i * page, page)
                for g in range(n_kv):
                    want_lo[pg, g], want_hi[pg, g] = PO.bounds_after(want_lo[pg, g], want_hi[pg, g], got_k[pg, g, lo:hi], lo > 0)
        assert int(pool.len[b]) == start[b] + n, why
    kept = ~touched.cuda()
    assert torch.equal(pool.k[kept], want_k[kept]) and torch.equal(pool.v[kept], want_v[kept]), why
    if want_lo is not None:
        assert np.array_equal(f64(pool.k_min), want_lo) and np.array_equal(f64(pool.k_max), want_hi), why


def snapshot(pool):
    return {m: getattr(pool, m).clone() for m in ("k", "v", "k_min", "k_max") if getattr(pool, m) is not None}


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("T", [1, 3, 70, 300])
@pytest.mark.parametrize("dtype,layout,rot,n_q,n_kv", [(torch.bfloat16, "half", 128, 28, 4), (torch.float32, "half", 48, 4, 1),
                                                       (torch.bfloat16, "interleaved", 64, 6, 3),
                                                       (torch.float32, "interleaved", 128, 32, 8)])
def test_append(rkv, page, T, dtype, layout, rot, n_q, n_kv):
    starts = [0, 1, page - 1, page, 127, 1000, 64, 130]
    B = len(starts)
    count = [T, max(T - 1, 0), T, 0, T, max(T // 2, 1), T, 1]
    pool = Pool(rkv, [s + T for s in starts], n_kv, page, T + page, lens=starts)
    ctx = rkv.Context(B, n_q, n_kv, 2048, 64)
    x = normal(gen(page + rot), B, T, (n_q + 2 * n_kv) * 128 + 64).to(dtype)[..., : (n_q + 2 * n_kv) * 128]   # strided rows
    q = torch.full((B, T, n_q, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    table = rkv.RopeTable(rot, 500000.0, layout, "bands", 8.0)
    before = snapshot(pool)
    ctx.paged_append(x, pool.struct(), table, q, count=i32(count))
    assert ctx.device_status() == 0
    f = QO.rope_frequencies(rot, 500000.0, "bands", 8.0)
    check_append(rkv, pool, x, starts, count, rot, layout, f, q, before)
    # once more, from given starts: what lay from there on is given up, and the bounds of a page kept in part stay
    again = [max(s - 5, 0) for s in starts]
    before = snapshot(pool)
    q.fill_(7)
    ctx.paged_append(x, pool.struct(), table, q, start=i32(again), count=i32(count))
    assert ctx.device_status() == 0
    check_append(rkv, pool, x, again, count, rot, layout, f, q, before)
    assert pool.len.tolist() == [a + c for a, c in zip(again, count)]


@pytest.mark.parametrize("page", [16, 128])
def test_append_without_rotation_or_bounds(rkv, page):
    B, T, n_q, n_kv = 3, 200, 4, 2
    pool = Pool(rkv, [400] * B, n_kv, page, 5, lens=[0, 33, 190], bounds=False)
    ctx = rkv.Context(B, n_q, n_kv, 512, 64)
    x = normal(gen(1), B, T, (n_q + 2 * n_kv) * 128).to(torch.bfloat16)
    q = torch.full((B, T, n_q, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    before = snapshot(pool)
    ctx.paged_append(x, pool.struct(), None, q)
    assert ctx.device_status() == 0
    check_append(rkv, pool, x, [0, 33, 190], [T] * B, 0, "half", None, q, before)
    assert torch.equal(q, x.view(B, T, -1, 128)[:, :, :n_q])


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append_in_chunks_is_append_at_once(rkv, page):
    n, n_q, n_kv = 1111, 8, 2
    ctx = rkv.Context(1, n_q, n_kv, 2048, 64)
    x = normal(gen(2), 1, n, (n_q + 2 * n_kv) * 128).to(torch.bfloat16)
    table = rkv.RopeTable()
    whole, parts = (Pool(rkv, [n], n_kv, page, 9) for _ in range(2))
    q = [torch.zeros((1, n, n_q, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx.paged_append(x, whole.struct(), table, q[0])
    at = 0
    for step in [1, 1, 14, 1, 100, 63, 1, 500, 64, 128, 238]:
        part = torch.zeros((1, step, n_q, 128), dtype=torch.bfloat16, device="cuda")
        ctx.paged_append(x[:, at: at + step], parts.struct(), table, part)
        q[1][:, at: at + step] = part
        at += step
    assert at == n and ctx.device_status() == 0 and parts.len.tolist() == [n]
    assert torch.equal(q[0], q[1])
    for m in ("k", "v", "k_min", "k_max"):
        assert torch.equal(getattr(whole, m), getattr(parts, m)), m


@pytest.mark.parametrize("what", ["overflow", "start behind the length", "negative start", "bad page", "count"])
def test_append_flags(rkv, what):
    page, T, n_q, n_kv = 16, 40, 2, 1
    pool = Pool(rkv, [64, 64], n_kv, page, 3, lens=[30, 10])
    ctx = rkv.Context(2, n_q, n_kv, 128, 64)
    x = normal(gen(4), 2, T, (n_q + 2 * n_kv) * 128).to(torch.bfloat16)
    q = torch.full((2, T, n_q, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    before = snapshot(pool)
    kw, bits, start, count = {}, 0, [30, 10], [T, T]
    if what == "overflow":                                   # 64 positions of room
        bits, count = rkv.DEV_APPEND_OVERFLOW, [34, T]
    elif what == "start behind the length":
        kw, bits, count = dict(start=i32([31, 10])), rkv.DEV_LEN_CLAMPED, [0, T]
    elif what == "negative start":
        kw, bits, count = dict(start=i32([-1, 10])), rkv.DEV_LEN_CLAMPED, [0, T]
    elif what == "count":                                    # below zero: none; above the rows given: those
        kw, count = dict(count=i32([-3, 1000])), [0, T]
    if what == "bad page":
        kept = pool.table.clone()
        pool.table[1, 1], pool.table[1, 2] = 10 ** 6, -1
        ctx.paged_append(x, pool.struct(), None, q, count=i32([5, T]))
        assert ctx.device_status() == rkv.DEV_BAD_INDEX and pool.len.tolist() == [35, 50]
        assert torch.equal(q[1], x.view(2, T, -1, 128)[1, :, :n_q])
        for i, rows in ((0, 6), (1, 0), (2, 0), (3, 2)):     # positions 10 .. 49
            lo = 10 if i == 0 else 0
            new = x.view(2, T, -1, 128)[1, 16 * i + lo - 10:, n_q][:rows]
            assert torch.equal(pool.k[kept[1, i], 0, lo: lo + rows], new)
            assert torch.equal(pool.k[kept[1, i], 0, lo + rows:], before["k"][kept[1, i], 0, lo + rows:])
        return
    if what == "overflow":
        kw = dict(count=i32([T, T]))
    ctx.paged_append(x, pool.struct(), None, q, **kw)
    assert ctx.device_status() == bits
    check_append(rkv, pool, x, start, count, 0, "half", None, q, before)
    assert pool.len.tolist() == [s + c for s, c in zip([30, 10], count)]


def test_append_of_keys_that_are_not_finite(rkv):
    """NaN does not enter the bounds, infinities do."""
    page, n_kv = 32, 1
    pool = Pool(rkv, [64], n_kv, page, 3)
    ctx = rkv.Context(1, 1, n_kv, 64, 64)
    x = normal(gen(4), 1, 40, 3 * 128).to(torch.bfloat16)
    x[0, 3, 128: 132] = torch.tensor([math.nan, math.inf, -math.inf, 0.0])
    x[0, 32:, 130] = math.nan
    q = torch.zeros((1, 40, 1, 128), dtype=torch.bfloat16, device="cuda")
    ctx.paged_append(x, pool.struct(), None, q)
    for i, rows in ((0, x[0, :32, 128: 256]), (1, x[0, 32:, 128: 256])):
        at = int(pool.table[0, i])
        lo, hi = PO.bounds_after(None, None, f64(rows), False)
        assert np.array_equal(f64(pool.k_min[at, 0]), lo) and np.array_equal(f64(pool.k_max[at, 0]), hi)


# ------------------------------------------------------------------------------------------------------------ attention
LENS = [0, 1, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 1000, 4097]


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n_q,n_kv", [(8, 1), (28, 4), (3, 3), (16, 8)])
def test_attention(rkv, page, n_q, n_kv):
    pool = Pool(rkv, [n + 1 for n in LENS], n_kv, page, page, lens=LENS, bounds=False)
    for b, n in enumerate(LENS):                 # rows behind the last one hold anything
        pg, r = PO.place(pool.table[b].tolist(), page, n)
        pool.k[pg, :, r:], pool.v[pg, :, r:] = math.nan, math.inf
    B = len(LENS)
    ctx = rkv.Context(B, n_q, n_kv, 5000, 64)
    q = normal(gen(7), B, n_q, 128).to(torch.bfloat16)
    active = i32([1] * B)
    active[4] = active[12] = 0
    for mask in (None, active):
        out = torch.full_like(q, 7.0)
        ctx.paged_attention(q, pool.struct(), out, active=mask)
        assert ctx.device_status() == 0
        for b, n in enumerate(LENS):
            if mask is not None and not int(mask[b]):
                assert (out[b] == 7).all()
                continue
            want, size = PO.attend(f64(q[b]), *pool.host(b, n))
            check_out(out[b], want, size, f"length {n}")


@pytest.mark.parametrize("n,hint", [(1, 0), (64, 64), (2000, 0), (9001, 0), (9001, 9001), (40000, 0)])
def test_attention_of_one_sequence(rkv, n, hint):
    n_q, n_kv = 8, 2
    pool = Pool(rkv, [n], n_kv, 64, n, lens=[n], bounds=False)
    ctx = rkv.Context(1, n_q, n_kv, 40960, 64)
    q = normal(gen(7), 1, n_q, 128).to(torch.bfloat16)
    out = torch.empty_like(q)
    ctx.paged_attention(q, pool.struct(), out, max_len_hint=hint)
    assert ctx.device_status() == 0
    check_out(out[0], *PO.attend(f64(q[0]), *pool.host(0, n)))


def test_attention_of_many_sequences(rkv):
    """More than the balanced form takes."""
    g = np.random.default_rng(3)
    lens = [int(x) for x in g.integers(0, 700, 300)]
    pool = Pool(rkv, [n + 1 for n in lens], 1, 32, 5, lens=lens, bounds=False)
    ctx = rkv.Context(300, 2, 1, 704, 64)
    q = normal(gen(7), 300, 2, 128).to(torch.bfloat16)
    out = torch.empty_like(q)
    ctx.paged_attention(q, pool.struct(), out)
    assert ctx.device_status() == 0
    for b, n in enumerate(lens):
        check_out(out[b], *PO.attend(f64(q[b]), *pool.host(b, n)), f"length {n}")


@pytest.mark.parametrize("n_kv,longest", [(2, 9001), (4, 4100), (8, 3000)])
def test_attention_of_a_batch_that_fills_the_chip(rkv, n_kv, longest):
    """Clusters whose CTAs have many tiles each, few for some sequences, none for others."""
    g = np.random.default_rng(n_kv)
    lens = [longest, 0, 1, 511, longest - 1] + [int(x) for x in g.integers(0, longest, 11)]
    pool = Pool(rkv, [n + 1 for n in lens], n_kv, 16, 5, lens=lens, bounds=False)
    ctx = rkv.Context(16, 3 * n_kv, n_kv, longest, 64)
    q = normal(gen(7), 16, 3 * n_kv, 128).to(torch.bfloat16)
    out = torch.empty_like(q)
    ctx.paged_attention(q, pool.struct(), out)
    assert ctx.device_status() == 0
    for b, n in enumerate(lens):
        check_out(out[b], *PO.attend(f64(q[b]), *pool.host(b, n)), f"length {n}")


def test_pool_beyond_32_bits(rkv):
    """Pages whose bytes lie beyond 2^32: rows are written there, attended and selected from there."""
    page, n_q, n_kv, n_pages, n = 128, 4, 2, 80000, 700       # 5.2 GB a buffer
    k, v = (torch.empty((n_pages, n_kv, page, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lo, hi = (torch.empty((n_pages, n_kv, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = i32([[n_pages - 1, n_pages - 3, 5, n_pages - 2, 0, n_pages - 9]])
    length = i32([0])
    c = rkv.paged_cache_struct(k, v, table, length, lo, hi)
    ctx = rkv.Context(1, n_q, n_kv, 1024, 64)
    x = normal(gen(1), 1, n, (n_q + 2 * n_kv) * 128).to(torch.bfloat16)
    q = torch.empty((1, n, n_q, 128), dtype=torch.bfloat16, device="cuda")
    ctx.paged_append(x, c, None, q)
    rows = f64(x[0]).reshape(n, n_q + 2 * n_kv, 128)
    kh, vh = (rows[:, a: a + n_kv].transpose(1, 0, 2) for a in (n_q, n_q + n_kv))
    last = q[:, -1].contiguous()
    out, near, idx = torch.empty_like(last), torch.empty_like(last), torch.zeros((1, n_kv, 3), dtype=torch.int32, device="cuda")
    ctx.paged_attention(last, c, out)
    ctx.paged_sparse_attention(last, c, 3, idx, near)
    assert ctx.device_status() == 0
    qh = f64(last[0])
    check_out(out[0], *PO.attend(qh, kh, vh))
    at = []
    for g in range(n_kv):
        held = [kh[g, i: i + page] for i in range(0, n, page)]
        s = PO.scores(qh[2 * g: 2 * g + 2], np.array([p.min(0) for p in held]), np.array([p.max(0) for p in held]))
        want = PO.select(s, 3, 1, 1)
        assert idx[0, g].tolist() == want
        at.append([p for i in want for p in range(i * page, min((i + 1) * page, n))])
    check_out(near[0], *PO.attend(qh, kh, vh, at=at))


@pytest.mark.parametrize("sparse", [False, True])
def test_attention_flags(rkv, sparse):
    """Pages that are not there are not attended, lengths above the table or the bound are cut; both set their flags."""
    page, n_q, n_kv = 16, 4, 2
    pool = Pool(rkv, [96, 96], n_kv, page, 3, lens=[96, 90])
    ctx = rkv.Context(2, n_q, n_kv, 128, 64)
    q = normal(gen(7), 2, n_q, 128).to(torch.bfloat16)
    host = [pool.host(0, 96), pool.host(1, 90)]

    def run(hint=0):
        out, idx = torch.full_like(q, 7.0), i32([[[7] * 6] * n_kv] * 2)
        if sparse:
            ctx.paged_sparse_attention(q, pool.struct(), 6, idx, out, max_len_hint=hint)
        else:
            ctx.paged_attention(q, pool.struct(), out, max_len_hint=hint)
        return out

    pool.len[0] = 200
    out = run()
    assert ctx.device_status() == rkv.DEV_LEN_CLAMPED
    for b in range(2):
        check_out(out[b], *PO.attend(f64(q[b]), *host[b]))
    pool.len[0] = 96
    out = run(hint=70)
    assert ctx.device_status() == rkv.DEV_LEN_CLAMPED
    for b in range(2):
        check_out(out[b], *PO.attend(f64(q[b]), *(x[:, :70] for x in host[b])))
    pool.table[1, 2], pool.table[1, 4] = -5, pool.k.shape[0]
    out = run()
    assert ctx.device_status() == rkv.DEV_BAD_INDEX
    check_out(out[0], *PO.attend(f64(q[0]), *host[0]))
    left = [p for p in range(90) if p // page not in (2, 4)]
    check_out(out[1], *PO.attend(f64(q[1]), *host[1], at=[left] * n_kv))
    pool.table[1] = -1
    out = run()
    assert ctx.device_status() == rkv.DEV_BAD_INDEX and (out[1] == 0).all()


# ------------------------------------------------------------------------------------------------------ shared prefixes
@pytest.mark.parametrize("together", [True, False])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("B,n_q,n_kv,prefix", [(2, 4, 4, 128), (5, 8, 1, 384), (20, 14, 2, 2048), (40, 7, 1, 1024),
                                               (17, 64, 8, 512), (3, 8, 2, 5120), (70, 8, 2, 768), (2, 2, 2, 128),
                                               (130, 8, 1, 256)])
def test_shared_prefix(rkv, page, B, n_q, n_kv, prefix, together):
    g = np.random.default_rng(B + page)
    lens = [prefix + int(x) for x in g.integers(0, 300, B)]
    lens[0] = prefix                              # nothing of its own
    lens[1] = prefix + 1
    if B > 4:
        lens[2], lens[3], lens[4] = 0, prefix - 1, prefix // 3      # shorter than the prefix
    pool = Pool(rkv, [max(n, prefix) + 1 for n in lens], n_kv, page, page + B, lens=lens, bounds=False, shared=prefix // page)
    for b, n in enumerate(lens):
        if n >= prefix:
            pg, r = PO.place(pool.table[b].tolist(), page, n)
            pool.k[pg, :, r:], pool.v[pg, :, r:] = math.nan, math.inf
    ctx = rkv.Context(B, n_q, n_kv, 6144, 64)
    if together:                                  # (by itself the library does so for longer prefixes)
        ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    q = normal(gen(7), B, n_q, 128).to(torch.bfloat16)
    q[B - 1] *= 12                                # one sequence whose attention is sharp
    active = torch.ones(B, dtype=torch.int32, device="cuda")
    active[B // 2] = 0
    for mask in (None, active):
        out = torch.full_like(q, 7.0)
        ctx.paged_attention(q, pool.struct(), out, active=mask, shared=pool.shared)
        assert ctx.device_status() == 0
        for b, n in enumerate(lens):
            if mask is not None and not int(mask[b]):
                assert (out[b] == 7).all()
                continue
            check_out(out[b], *PO.attend(f64(q[b]), *pool.host(b, n)), f"sequence {b} of length {n}")


def test_shared_prefix_that_the_library_reads_once(rkv):
    """Long enough for one pass over it; queries far from the origin, whose maxima grow along the prefix."""
    page, B, n_q, n_kv, prefix = 64, 10, 28, 4, 16384
    lens = [prefix + 50 * b for b in range(B)]
    pool = Pool(rkv, lens, n_kv, page, 8, lens=lens, bounds=False, shared=prefix // page)
    for i in range(prefix // page):               # keys that get louder
        pool.k[int(pool.shared[i])] *= 0.2 + 2.0 * i * page / prefix
    ctx = rkv.Context(B, n_q, n_kv, 17408, 64)
    q = (normal(gen(7), B, n_q, 128) * 3).to(torch.bfloat16)
    before, out = ctx.launch_count, torch.empty_like(q)
    ctx.paged_attention(q, pool.struct(), out, shared=pool.shared)
    assert ctx.launch_count - before == 3 and ctx.device_status() == 0
    for b in (0, 1, B - 1):
        check_out(out[b], *PO.attend(f64(q[b]), *pool.host(b, lens[b])))


def test_shared_pages_that_are_not_there(rkv):
    page, B, n_q, n_kv, prefix = 32, 6, 4, 2, 512
    lens = [prefix + 10 * b for b in range(B)]
    pool = Pool(rkv, lens, n_kv, page, 8, lens=lens, bounds=False, shared=prefix // page)
    host = [pool.host(b, n) for b, n in enumerate(lens)]
    ctx = rkv.Context(B, n_q, n_kv, 1024, 64)
    ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    q = normal(gen(7), B, n_q, 128).to(torch.bfloat16)
    out = torch.empty_like(q)
    shared = pool.shared.clone()
    shared[3], shared[7] = -1, 10 ** 8
    pool.table[:, 3], pool.table[:, 7] = -1, 10 ** 8
    ctx.paged_attention(q, pool.struct(), out, shared=shared)
    assert ctx.device_status() == rkv.DEV_BAD_INDEX
    for b, n in enumerate(lens):
        left = [p for p in range(n) if p // page not in (3, 7)]
        check_out(out[b], *PO.attend(f64(q[b]), *host[b], at=[left] * n_kv))


# ------------------------------------------------------------------------------------------------------- selected pages
def check_sparse(rkv, ctx, pool, q, lens, top, first, last, active=None, hint=0):
    B, n_q = q.shape[:2]
    n_kv, page = pool.n_kv, pool.page
    out, idx = torch.full_like(q, 7.0), torch.full((B, n_kv, top), -7, dtype=torch.int32, device="cuda")
    ctx.paged_sparse_attention(q, pool.struct(), top, idx, out, active=active, first_pages=first, last_pages=last,
                               max_len_hint=hint)
    assert ctx.device_status() == 0
    lo, hi, G = f64(pool.k_min), f64(pool.k_max), n_q // n_kv
    for b, n in enumerate(lens):
        if active is not None and not int(active[b]):
            assert (out[b] == 7).all() and (idx[b] == -7).all()
            continue
        at = []
        for g in range(n_kv):
            t = pool.table[b, : -(-n // page)].long().cpu().numpy()
            s = PO.scores(f64(q[b, g * G: (g + 1) * G]), lo[t, g], hi[t, g])
            want = PO.select(s, top, first, last)
            assert idx[b, g].tolist() == want + [-1] * (top - len(want)), f"sequence {b} of length {n}, head {g}"
            at.append([p for i in want for p in range(i * page, min((i + 1) * page, n))])
        check_out(out[b], *PO.attend(f64(q[b]), *pool.host(b, n), at=at), f"sequence {b} of length {n}")


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n_q,n_kv", [(8, 1), (28, 4), (2, 2)])
@pytest.mark.parametrize("top,first,last", [(1, 1, 1), (3, 0, 0), (7, 2, 3), (40, 1, 1), (4, 5, 9), (300, 0, 1)])
def test_sparse(rkv, page, n_q, n_kv, top, first, last):
    pool = Pool(rkv, [n + 1 for n in LENS], n_kv, page, page + top, lens=LENS)
    for b, n in enumerate(LENS):                 # rows behind the last one hold anything
        pg, r = PO.place(pool.table[b].tolist(), page, n)
        pool.k[pg, :, r:], pool.v[pg, :, r:] = math.nan, math.inf
    B = len(LENS)
    ctx = rkv.Context(B, n_q, n_kv, 5000, 64)
    q = normal(gen(7), B, n_q, 128).to(torch.bfloat16)
    active = i32([1] * B)
    active[4] = active[12] = 0
    check_sparse(rkv, ctx, pool, q, LENS, top, first, last)
    check_sparse(rkv, ctx, pool, q, LENS, top, first, last, active=active)


@pytest.mark.parametrize("n,page,top", [(327680, 16, 512), (131072, 64, 64), (70001, 16, 33), (20000, 128, 150)])
def test_sparse_of_a_long_sequence(rkv, n, page, top):
    pool = Pool(rkv, [n], 1, page, n % 97, lens=[n])
    ctx = rkv.Context(1, 4, 1, 327680, 64)
    q = normal(gen(3), 1, 4, 128).to(torch.bfloat16)
    check_sparse(rkv, ctx, pool, q, [n], top, 1, 1)
    check_sparse(rkv, ctx, pool, q, [n], top, 1, 1, hint=n)


@pytest.mark.parametrize("n_q", [4, 16])
@pytest.mark.parametrize("top", [500, 600])
def test_sparse_of_many_pages_in_a_batch(rkv, top, n_q):
    """About as many pages as the attention's CTAs pick themselves; a batch that fills the chip."""
    lens = [9600, 9601, 9700, 0, 3, 8000, 8001, 9599] * 2
    pool = Pool(rkv, [n + 1 for n in lens], 2, 16, top, lens=lens)
    ctx = rkv.Context(16, n_q, 2, 9728, 64)
    q = normal(gen(8), 16, n_q, 128).to(torch.bfloat16)
    check_sparse(rkv, ctx, pool, q, lens, top, 1, 1)


@pytest.mark.parametrize("how", ["all alike", "pairs", "two kinds", "zero query", "extremes", "infinite"])
def test_sparse_ties(rkv, how):
    """Pages of equal scores: the lower ones.  Scores of very different size, infinities in bounds and queries."""
    page, P, n_kv, top = 16, 700, 2, 300
    n = P * page - 3
    pool = Pool(rkv, [n], n_kv, page, 11, lens=[n])
    q = normal(gen(3), 1, 8, 128).to(torch.bfloat16)
    at = pool.table[0].long()
    if how == "all alike":
        pool.k_min[:], pool.k_max[:] = -1.0, 1.0
    elif how == "pairs":
        pool.k_min[at[1::2]], pool.k_max[at[1::2]] = pool.k_min[at[0::2]], pool.k_max[at[0::2]]
    elif how == "two kinds":
        pool.k_min[at], pool.k_max[at] = -1.0, 1.0
        pool.k_max[at[5::7]] = 2.0
    elif how == "zero query":
        q.zero_()
    elif how == "extremes":                      # down to subnormals, up to the largest
        s = torch.exp2(torch.linspace(-130, 126, P, device="cuda"))[:, None, None]
        pool.k_min[at], pool.k_max[at] = (-s).to(torch.bfloat16), s.to(torch.bfloat16)
    else:
        pool.k_max[at[17], :, 5], pool.k_min[at[18], :, 6] = math.inf, -math.inf
        q[0, 1, 9] = -math.inf
        q[0, 5, 5] = math.inf
    ctx = rkv.Context(1, 8, n_kv, 16384, 64)
    out, idx = torch.empty_like(q), torch.empty((1, n_kv, top), dtype=torch.int32, device="cuda")
    ctx.paged_sparse_attention(q, pool.struct(), top, idx, out)
    for g in range(n_kv):
        s = PO.scores(f64(q[0, 4 * g: 4 * g + 4]), f64(pool.k_min[at, g]), f64(pool.k_max[at, g]))
        assert idx[0, g].tolist() == PO.select(s, top, 1, 1)
    if how != "infinite":
        pos = [[p for i in idx[0, g].tolist() for p in range(i * page, min((i + 1) * page, n))] for g in range(n_kv)]
        check_out(out[0], *PO.attend(f64(q[0]), *pool.host(0, n), at=pos))


# --------------------------------------------------------------------------------------------------------- calls as used
def test_prompt_tokens_and_both_attentions(rkv):
    """A ragged batch behind a common prompt: the prompt is appended once, its pages are in every table, then prompts of
    their own and tokens follow, each attended in full and over selected pages."""
    B, n_q, n_kv, page, prefix = 4, 8, 2, 32, 256
    G, f = n_q // n_kv, QO.rope_frequencies(128, 10000.0)
    pool = Pool(rkv, [600] * B, n_kv, page, 21, lens=[0] * B, shared=prefix // page)
    table, g = rkv.RopeTable(128, 10000.0), gen(5)
    one, ctx = rkv.Context(1, n_q, n_kv, 640, 64), rkv.Context(B, n_q, n_kv, 640, 64)
    ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    width = (n_q + 2 * n_kv) * 128
    xs = [normal(g, 1, prefix, width).to(torch.bfloat16)]
    head = rkv.paged_cache_struct(pool.k, pool.v, pool.table[:1, : prefix // page].contiguous(), i32([0]), pool.k_min, pool.k_max)
    q = torch.empty((1, prefix, n_q, 128), dtype=torch.bfloat16, device="cuda")
    one.paged_append(xs[0], head, table, q)
    pool.len.fill_(prefix)
    hist = [[f64(xs[0][0])] for _ in range(B)]
    cache = pool.struct()
    count = [100, 0, 33, 1]
    x = normal(g, B, 100, width).to(torch.bfloat16)
    q = torch.empty((B, 100, n_q, 128), dtype=torch.bfloat16, device="cuda")
    ctx.paged_append(x, cache, table, q, count=i32(count))
    for b in range(B):
        hist[b].append(f64(x[b, : count[b]]))
    for step in range(6):
        x = normal(g, B, 1, width)
        q = torch.empty((B, 1, n_q, 128), dtype=torch.bfloat16, device="cuda")
        out, near = torch.empty((B, n_q, 128), dtype=torch.bfloat16, device="cuda"), None
        ctx.paged_append(x, cache, table, q)
        ctx.paged_attention(q.view(B, n_q, 128), cache, out, shared=pool.shared)
        near, idx = torch.empty_like(out), torch.empty((B, n_kv, 5), dtype=torch.int32, device="cuda")
        ctx.paged_sparse_attention(q.view(B, n_q, 128), cache, 5, idx, near)
        assert ctx.device_status() == 0 and one.device_status() == 0
        for b in range(B):
            hist[b].append(f64(x[b]))
            n = prefix + count[b] + step + 1
            assert int(pool.len[b]) == n
            rows = np.concatenate(hist[b]).reshape(n, n_q + 2 * n_kv, 128)
            k = QO.rope(rows[:, n_q: n_q + n_kv], np.arange(n), *f, "half")
            got_k, got_v = pool.host(b, n)
            assert (np.abs(got_k.transpose(1, 0, 2) - k) <= 2.0 ** -8 * np.abs(k) + 2.0 ** -14).all()
            assert (np.abs(got_v.transpose(1, 0, 2) - rows[:, n_q + n_kv:]) <= 2.0 ** -8 * np.abs(rows[:, n_q + n_kv:])).all()
            check_out(out[b], *PO.attend(f64(q[b, 0]), got_k, got_v), f"step {step}, sequence {b}")
            at = []
            for h in range(n_kv):
                pages = [got_k[h, i: i + page] for i in range(0, n, page)]        # the bounds, from the stored keys
                s = PO.scores(f64(q[b, 0, h * G: (h + 1) * G]), np.array([p.min(0) for p in pages]), np.array([p.max(0) for p in pages]))
                want = PO.select(s, 5, 1, 1)
                assert idx[b, h].tolist() == want
                at.append([p for i in want for p in range(i * page, min((i + 1) * page, n))])
            check_out(near[b], *PO.attend(f64(q[b, 0]), got_k, got_v, at=at), f"step {step}, sequence {b}")


def test_captured_and_replayed_on_one_workspace(rkv):
    """Two graphs of a whole step on one context, replayed in turn on a side stream while lengths grow on the device, give
    what the eager calls on a context of their own give."""
    B, n_q, n_kv, page, prefix, top = 3, 8, 2, 16, 128, 6
    side, table = torch.cuda.Stream(), rkv.RopeTable()
    shared, own = (rkv.Context(B, n_q, n_kv, 1024, 64) for _ in range(2))
    for ctx in (shared, own):
        ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    width, steps = (n_q + 2 * n_kv) * 128, []
    for seed in (1, 2):
        pools = [Pool(rkv, [700, 300, 900], n_kv, page, seed, lens=[140, 128, 500], shared=prefix // page) for _ in range(2)]
        x = normal(gen(seed), B, 1, width)
        bufs = [(torch.zeros((B, 1, n_q, 128), dtype=torch.bfloat16, device="cuda"),
                 torch.zeros((B, n_q, 128), dtype=torch.bfloat16, device="cuda"),
                 torch.zeros((B, n_q, 128), dtype=torch.bfloat16, device="cuda"),
                 torch.zeros((B, n_kv, top), dtype=torch.int32, device="cuda")) for _ in range(2)]

        def step(ctx, i, x=x, pools=pools, bufs=bufs, cs=[p.struct() for p in pools]):
            q, out, near, idx = bufs[i]
            ctx.paged_append(x, cs[i], table, q)
            ctx.paged_attention(q.view(B, n_q, 128), cs[i], out, shared=pools[i].shared)
            ctx.paged_sparse_attention(q.view(B, n_q, 128), cs[i], top, idx, near)

        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            step(shared, 0)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step(shared, 0)
        step(own, 1)
        torch.cuda.synchronize()
        steps.append((graph, step, x, pools, bufs))
    for rep in range(12):
        for graph, step, x, pools, bufs in steps:
            x.copy_(normal(gen(100 + rep), *x.shape))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for graph, *_ in steps:
                graph.replay()
        for _, step, *_ in steps:
            step(own, 1)
        torch.cuda.synchronize()
        for _, _, _, pools, bufs in steps:
            for a, b in zip(*bufs):
                assert torch.equal(a, b)
            for m in ("k", "v", "k_min", "k_max", "len"):
                assert torch.equal(getattr(pools[0], m), getattr(pools[1], m))
    assert shared.device_status() == 0 and own.device_status() == 0


def test_results_do_not_depend_on_the_run(rkv):
    B, n_q, n_kv, page, prefix = 9, 28, 4, 64, 1024
    lens = [prefix + 97 * b for b in range(B)]
    pool = Pool(rkv, lens, n_kv, page, 3, lens=lens, shared=prefix // page)
    ctx = rkv.Context(B, n_q, n_kv, 2048, 64)
    ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    q = normal(gen(7), B, n_q, 128).to(torch.bfloat16)
    first = None
    for _ in range(5):
        out, near, idx = torch.empty_like(q), torch.empty_like(q), i32([[[0] * 7] * n_kv] * B)
        ctx.paged_attention(q, pool.struct(), out, shared=pool.shared)
        ctx.paged_sparse_attention(q, pool.struct(), 7, idx, near)
        first = first or (out, near, idx)
        for a, b in zip(first, (out, near, idx)):
            assert torch.equal(a, b)


def test_paged_calls_and_a_pending_selection(rkv):
    """The attention calls use the workspace that a full attention has left its logits in: the selection behind is refused."""
    from paper_2411_05787_b200 import synth
    c = synth.alloc_cache([256], [200], 2, torch.device("cuda"), fill=0.0)
    cs = rkv.cache_struct(c.k, c.v, c.row_offset, c.cap, c.len)
    ctx = rkv.Context(1, 4, 2, 256, 64)
    pool = Pool(rkv, [100], 2, 16, 1, lens=[100])
    q = normal(gen(7), 1, 4, 128).to(torch.bfloat16)
    out, idx = torch.empty_like(q), torch.zeros((1, 2, 8), dtype=torch.int32, device="cuda")
    ctx.full_attention(q, cs, out)
    ctx.select_topk(q, cs, i32([8]), 8, idx)
    for call in (lambda: ctx.paged_attention(q, pool.struct(), out), lambda: ctx.paged_sparse_attention(q, pool.struct(), 8, idx, out)):
        ctx.full_attention(q, cs, out)
        call()
        with pytest.raises(rkv.RkvError):
            ctx.select_topk(q, cs, i32([8]), 8, idx)
    assert ctx.device_status() == 0


def test_packed_attention_right_behind_a_paged_append(rkv):
    """With one KV head and a table in order, a pool's rows are a packed cache's.  The packed attention behind an append may
    request its first tiles ahead only of launches that leave the cache alone, which this one does not."""
    n, group, page = 4096, 4, 64
    pool = Pool(rkv, [n], 1, page, 1, spare=0)
    pool.table[0] = torch.arange(n // page)
    rows = [x.view(n, 128) for x in (pool.k, pool.v)]
    off, cap = torch.zeros(1, dtype=torch.int64, device="cuda"), i32([n])
    cs, ps = rkv.cache_struct(*rows, off, cap, pool.len), pool.struct()
    ctx, table, g = rkv.Context(1, group, 1, n, 64), rkv.RopeTable(), gen(3)
    q = torch.empty((1, n, group, 128), dtype=torch.bfloat16, device="cuda")
    xs = [(normal(g, 1, n, (group + 2) * 128) * s).to(torch.bfloat16) for s in (1.0, 2.0, 0.5)]

    def run(x, wait):
        ctx.paged_append(x, ps, table, q, start=i32([0]))
        if wait:
            torch.cuda.synchronize()
        out = torch.empty((1, group, 128), dtype=torch.bfloat16, device="cuda")
        ctx.full_attention(q[0, -1:], cs, out)
        return out

    want = [run(x, True) for x in xs]
    got = [run(x, False) for _ in range(20) for x in xs]
    for i, out in enumerate(got):
        assert torch.equal(out, want[i % 3])
    assert ctx.device_status() == 0


def test_refusals_of_the_library(rkv):
    pool = Pool(rkv, [100], 2, 16, 1, lens=[100])
    ctx = rkv.Context(1, 4, 2, 256, 64)
    q = torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda")
    out, idx = torch.empty_like(q), torch.zeros((1, 2, 8), dtype=torch.int32, device="cuda")
    for kw in (dict(first_pages=-1), dict(last_pages=-1), dict(max_len_hint=257), dict(max_len_hint=-1)):
        with pytest.raises(rkv.RkvError):
            ctx.paged_sparse_attention(q, pool.struct(), 8, idx, out, **kw)
    with pytest.raises(rkv.RkvError):
        ctx.paged_sparse_attention(q, pool.struct(), 0, idx[..., :0].contiguous(), out)
    with pytest.raises(rkv.RkvError):
        ctx.paged_attention(q, pool.struct(), out, max_len_hint=300)
    with pytest.raises(rkv.RkvError):
        ctx.set_option(rkv.OPT_SHARED_MIN, -1)
    assert ctx.get_option(rkv.OPT_SHARED_MIN) == 1 << 19
    with pytest.raises(ValueError):              # more shared pages than the table has room for
        ctx.paged_attention(q, pool.struct(), out, shared=torch.zeros(8, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        ctx.paged_attention(q, pool.struct(), out, shared=torch.zeros(2, dtype=torch.int64, device="cuda"))
    pool.k_min = pool.k_max = None
    with pytest.raises(ValueError):              # no bounds to select by
        ctx.paged_sparse_attention(q, pool.struct(), 8, idx, out)
    ctx.paged_attention(q, pool.struct(), out)
    assert ctx.device_status() == 0
