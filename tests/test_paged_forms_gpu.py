"""Forms of the paged cache's kernels that batches of special shapes reach, against the definition in 64 bits (tolerances as in
test_paged_gpu.py)."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from test_paged_gpu import Pool, check_out, check_sparse, f64, gen, i32, normal, rkv  # noqa: F401  (rkv: the fixture)

pytestmark = pytest.mark.gpu


def attend64(q, pool, b, n, gone=(), scale=1.0 / math.sqrt(128)):
    """out and sum_j p_j |v_j| [Hq, 128] of sequence b over its first n positions but those of the pages `gone`."""
    n_kv, page = pool.n_kv, pool.page
    some = [i for i in range(-(-n // page)) if i not in gone]
    if not some:
        return (np.zeros(q.shape),) * 2
    at = torch.tensor(some, device="cuda")
    pos = (at[:, None] * page + torch.arange(page, device="cuda")).flatten()
    k, v = (x[pool.pages[b, at].long()].double().transpose(0, 1).flatten(1, 2)[:, pos < n] for x in (pool.k, pool.v))
    s = q.double().view(n_kv, -1, 128) @ k.transpose(1, 2) * scale
    p = torch.softmax(s, -1)
    return tuple(f64((p @ x).reshape(q.shape)) for x in (v, v.abs()))


def splits_of(ctx_len, n_seq, n_q, n_kv, prefix):
    """CTAs that share a prefix, per KV head and 256 rows."""
    blocks = -(-n_seq * (n_q // n_kv) // 256) * n_kv
    most = min(-(-ctx_len // 64), 128)
    return max(min(torch.cuda.get_device_properties(0).multi_processor_count // blocks, -(-prefix // 64), most // 2), 1)


def behind_prefix(rkv, B, n_q, n_kv, page, prefix, longest, seed, gone=(), scale=0.0, louder=True, loud=3.0):
    """A batch behind a prefix whose keys get louder (maxima grow from tile to tile), pages `gone` missing from it."""
    g = np.random.default_rng(seed)
    lens = [prefix + int(x) for x in g.integers(0, longest, B)]
    lens[0], lens[1] = prefix, prefix + 1
    if B > 4:
        lens[2], lens[3] = 0, prefix - 1          # shorter than the prefix
    pool = Pool(rkv, [max(n, prefix) for n in lens], n_kv, page, seed, lens=lens, bounds=False, shared=prefix // page)
    if louder:
        grows = 0.2 + 2.0 * torch.arange(prefix // page, device="cuda") * page / prefix
        pool.k[pool.shared.long()] *= grows.to(torch.bfloat16)[:, None, None, None]
    pool.pages = pool.table.clone()
    shared = pool.shared.clone()
    for n, i in enumerate(gone):
        shared[i] = pool.table[:, i] = -1 if n % 2 else 10 ** 8
    ctx = rkv.Context(B, n_q, n_kv, max(lens), 64, softmax_scale=scale)
    ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    q = (normal(gen(seed), B, n_q, 128) * loud).to(torch.bfloat16)
    out, before = torch.full_like(q, 7.0), ctx.launch_count
    ctx.paged_attention(q, pool.struct(), out, shared=shared)
    assert ctx.launch_count - before == 3
    assert ctx.device_status() == (rkv.DEV_BAD_INDEX if len(gone) else 0)
    for b, n in enumerate(lens):
        want = attend64(q[b], pool, b, n, gone, scale or 1.0 / math.sqrt(128))
        check_out(out[b], *want, f"sequence {b} of length {n}")


@pytest.mark.parametrize("B,n_q,n_kv,page,prefix", [(40, 28, 4, 64, 16384), (40, 28, 4, 16, 16384), (37, 28, 4, 128, 16384),
                                                    (64, 4, 1, 64, 64 * 64 * 13), (33, 24, 6, 32, 24576)])
def test_two_blocks_of_rows_and_many_tiles(rkv, B, n_q, n_kv, page, prefix):
    """More than 128 rows a head, and more tiles to a CTA than its ring and its buffers hold: blocks of 256, of 256 and
    a ragged one of fewer than 128, of 128 and a few."""
    assert B * (n_q // n_kv) > 128
    assert prefix // 64 >= 12 * splits_of(prefix + 300, B, n_q, n_kv, prefix)
    behind_prefix(rkv, B, n_q, n_kv, page, prefix, 300, B + page)


@pytest.mark.parametrize("B", [6, 40])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_missing_shared_pages_by_the_tile(rkv, B, page):
    """Tiles of a CTA that are missing or have holes: its first, one in the middle, its last, all of them; one block of rows
    and two."""
    n_q, n_kv, prefix = 28, 4, 16384
    n_cta = splits_of(prefix + 200, B, n_q, n_kv, prefix)
    tiles = prefix // 64
    dead = {0, 3, 5 + 2 * n_cta, 7 + n_cta, tiles - 1} | set(range(9, tiles, n_cta))
    gone = sorted({p for t in dead for p in range(t * 64 // page, max((t + 1) * 64 // page, t * 64 // page + 1))})
    if page == 16:
        gone += [4 * (12 + n_cta) + 1, 4 * 14, 4 * (15 + n_cta) + 3]     # a part of a tile
    behind_prefix(rkv, B, n_q, n_kv, page, prefix, 200, B + page, gone=gone)


@pytest.mark.parametrize("n_q", [1, 2])
def test_a_prefix_of_more_sequences_than_the_balanced_form_takes(rkv, n_q):
    behind_prefix(rkv, 300, n_q, 1, 32, 1024, 400, 9)


@pytest.mark.parametrize("scale", [0.3, 0.004])
def test_softmax_scale(rkv, scale):
    loud = 0.3 if scale > 0.1 else 6.0            # |scores| of tens at most
    behind_prefix(rkv, 24, 14, 2, 64, 4096, 300, 5, scale=scale, loud=loud)
    lens = [0, 1, 1000, 3000]
    pool = Pool(rkv, [n + 1 for n in lens], 2, 32, 6, lens=lens)
    pool.pages = pool.table
    ctx = rkv.Context(4, 8, 2, 4096, 64, softmax_scale=scale)
    q = (normal(gen(3), 4, 8, 128) * loud).to(torch.bfloat16)
    out, near, idx = torch.empty_like(q), torch.empty_like(q), i32([[[0] * 9] * 2] * 4)
    ctx.paged_attention(q, pool.struct(), out)
    ctx.paged_sparse_attention(q, pool.struct(), 9, idx, near)
    assert ctx.device_status() == 0
    for b, n in enumerate(lens):
        check_out(out[b], *attend64(q[b], pool, b, n, scale=scale), f"length {n}")
        at = [[p for i in idx[b, g].tolist() if i >= 0 for p in range(i * 32, min((i + 1) * 32, n))] for g in range(2)]
        check_out(near[b], *PO.attend(f64(q[b]), *pool.host(b, n), at=at, scale=scale), f"length {n}, selected")


def test_one_long_sequence_among_short_ones(rkv):
    """A head with more tiles than there are slots for its partials: fewer CTAs, longer runs."""
    lens = [40000, 5, 700, 0, 64, 129, 1, 300]
    pool = Pool(rkv, [n + 1 for n in lens], 4, 64, 3, lens=lens, bounds=False)
    pool.pages = pool.table
    ctx = rkv.Context(8, 28, 4, 40960, 64)
    q = normal(gen(5), 8, 28, 128).to(torch.bfloat16)
    out, before = torch.empty_like(q), ctx.launch_count
    ctx.paged_attention(q, pool.struct(), out)
    assert ctx.device_status() == 0 and ctx.launch_count - before == 2
    for b, n in enumerate(lens):
        check_out(out[b], *attend64(q[b], pool, b, n), f"length {n}")


@pytest.mark.parametrize("own", [-1, 9000])
def test_one_long_sequence_behind_a_prefix(rkv, own):
    """The same where slots are taken by the prefix: a sequence that just misses a prefix of more tiles than slots are left
    and attends all of it by itself; one that has as many of its own."""
    B, n_q, n_kv, page, prefix = 6, 8, 2, 64, 64 * 140
    lens = [prefix + x for x in (own, 3, 0, 70, 200, 1)]
    pool = Pool(rkv, [max(n, prefix) for n in lens], n_kv, page, 3, lens=lens, bounds=False, shared=prefix // page)
    pool.pages = pool.table
    ctx = rkv.Context(B, n_q, n_kv, 18432, 64)
    ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    q = normal(gen(5), B, n_q, 128).to(torch.bfloat16)
    out, before = torch.empty_like(q), ctx.launch_count
    ctx.paged_attention(q, pool.struct(), out, shared=pool.shared)
    assert ctx.device_status() == 0 and ctx.launch_count - before == 3
    for b, n in enumerate(lens):
        check_out(out[b], *attend64(q[b], pool, b, n), f"length {n}")


# ------------------------------------------------------------------------------------- scores of groups of five to eight
@pytest.mark.parametrize("G", [5, 7, 8])
@pytest.mark.parametrize("how", ["all alike", "pairs", "two kinds", "zero query", "extremes", "infinite"])
def test_ties_and_extremes_of_large_groups(rkv, how, G):
    page, P, n_kv, top = 16, 700, 2, 300
    n = P * page - 3
    pool = Pool(rkv, [n], n_kv, page, 11, lens=[n])
    q = normal(gen(3), 1, G * n_kv, 128).to(torch.bfloat16)
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
    elif how == "extremes":                       # down to subnormals, up to the largest
        s = torch.exp2(torch.linspace(-130, 126, P, device="cuda"))[:, None, None]
        pool.k_min[at], pool.k_max[at] = (-s).to(torch.bfloat16), s.to(torch.bfloat16)
    else:
        pool.k_max[at[17], :, 5], pool.k_min[at[18], :, 6] = math.inf, -math.inf
        q[0, 1, 9] = -math.inf
        q[0, G + 1, 5] = math.inf
    ctx = rkv.Context(1, G * n_kv, n_kv, 16384, 64)
    out, idx = torch.empty_like(q), torch.empty((1, n_kv, top), dtype=torch.int32, device="cuda")
    ctx.paged_sparse_attention(q, pool.struct(), top, idx, out)
    assert ctx.device_status() == 0
    for g in range(n_kv):
        s = PO.scores(f64(q[0, G * g: G * (g + 1)]), f64(pool.k_min[at, g]), f64(pool.k_max[at, g]))
        assert idx[0, g].tolist() == PO.select(s, top, 1, 1)
    if how != "infinite":
        pos = [[p for i in idx[0, g].tolist() for p in range(i * page, min((i + 1) * page, n))] for g in range(n_kv)]
        check_out(out[0], *PO.attend(f64(q[0]), *pool.host(0, n), at=pos))


@pytest.mark.parametrize("G", [5, 8])
def test_pages_that_are_not_there_come_last_in_large_groups(rkv, G):
    page, n_kv, top = 16, 2, 6
    pool = Pool(rkv, [400, 90], n_kv, page, 3, lens=[400, 90])
    ctx = rkv.Context(2, G * n_kv, n_kv, 512, 64)
    q = normal(gen(7), 2, G * n_kv, 128).to(torch.bfloat16)
    host, kept = [pool.host(0, 400), pool.host(1, 90)], pool.table.clone()
    pool.table[0, 3], pool.table[0, 20], pool.table[1, 2], pool.table[1, 4] = -1, 10 ** 8, -5, pool.k.shape[0]
    out, idx = torch.empty_like(q), torch.empty((2, n_kv, top), dtype=torch.int32, device="cuda")
    ctx.paged_sparse_attention(q, pool.struct(), top, idx, out)
    assert ctx.device_status() == rkv.DEV_BAD_INDEX
    lo, hi = f64(pool.k_min), f64(pool.k_max)
    for b, (n, gone) in enumerate(((400, (3, 20)), (90, (2, 4)))):
        at = []
        for g in range(n_kv):
            t = kept[b, : -(-n // page)].long().cpu().numpy()
            s = PO.scores(f64(q[b, g * G: (g + 1) * G]), lo[t, g], hi[t, g])
            s[list(gone)] = -math.inf
            want = PO.select(s, top, 1, 1)
            assert idx[b, g].tolist() == want
            at.append([p for i in want if i not in gone for p in range(i * page, min((i + 1) * page, n))])
        check_out(out[b], *PO.attend(f64(q[b]), *host[b], at=at))


@pytest.mark.parametrize("G", [5, 6, 8])
def test_ragged_batch_of_large_groups(rkv, G):
    lens = [0, 1, 33, 4097, 31, 32, 2000, 700]
    pool = Pool(rkv, [n + 1 for n in lens], 3, 32, G, lens=lens)
    ctx = rkv.Context(8, 3 * G, 3, 4608, 64)
    q = normal(gen(8), 8, 3 * G, 128).to(torch.bfloat16)
    active = i32([1, 1, 1, 1, 0, 1, 1, 1])
    check_sparse(rkv, ctx, pool, q, lens, 11, 1, 1, active=active)


# ------------------------------------------------------------------------------------------------------ inactive sequences
@pytest.mark.parametrize("G", [4, 7])
@pytest.mark.parametrize("form", ["clusters", "balanced", "shared"])
def test_inactive_sequences_may_hold_anything(rkv, form, G):
    """Queries of NaN, lengths and tables of garbage where the mask is zero: no flag, outputs left alone, the others as ever."""
    n_kv, page, prefix = 2, 64, 1024
    lens = [prefix + x for x in ((100, 0, 700, 31, 5) if form != "balanced" else (9000, 0, 3, 8000, 1))]
    B = len(lens)
    pool = Pool(rkv, lens, n_kv, page, G, lens=lens, shared=prefix // page)
    pool.pages = pool.table.clone()
    ctx = rkv.Context(B, G * n_kv, n_kv, 32768 if form == "balanced" else 2048, 64)
    ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    q = normal(gen(2), B, G * n_kv, 128).to(torch.bfloat16)
    active = i32([1, 0, 1, 0, 0])
    q[1], q[3], q[4] = math.nan, math.inf, -math.inf
    pool.len[1], pool.len[3], pool.len[4] = 2 ** 31 - 1, -7, prefix
    pool.table[1], pool.table[3], pool.table[4] = 10 ** 9, -(10 ** 9), -1
    out, near, idx = torch.full_like(q, 7.0), torch.full_like(q, 7.0), i32([[[-7] * 9] * n_kv] * B)
    ctx.paged_attention(q, pool.struct(), out, active=active, shared=pool.shared if form == "shared" else None)
    ctx.paged_sparse_attention(q, pool.struct(), 9, idx, near, active=active)
    assert ctx.device_status() == 0
    for b, n in enumerate(lens):
        if not int(active[b]):
            assert (out[b] == 7).all() and (near[b] == 7).all() and (idx[b] == -7).all()
            continue
        check_out(out[b], *attend64(q[b], pool, b, n), f"length {n}")
        at = [[p for i in idx[b, g].tolist() if i >= 0 for p in range(i * page, min((i + 1) * page, n))] for g in range(n_kv)]
        check_out(near[b], *PO.attend(f64(q[b]), *pool.host(b, n), at=at), f"length {n}, selected")
