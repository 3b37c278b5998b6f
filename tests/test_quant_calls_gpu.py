"""The 8-bit cache's calls where they meet other calls: lengths read while they are about to change, workspaces that an
earlier call has left its traces in, sequences that one call refuses and the next one reads."""
import numpy as np
import pytest
import torch

from oracle import rkv_oracle as O
from test_quant_gpu import (Host, check_out, check_scores, context, f64, filled, gen, head_rows, i32, normal, reference as
                            quant_reference, struct)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2411_05787_b200 import rkv, runner, synth
    return rkv, runner, synth


# ---------------------------------------------------------------------------------------------------------------- store
@pytest.mark.parametrize("given", ["append", "lengths as start"])
def test_store_reads_lengths_before_they_change(mods, given):
    """Padded batches with CTAs that have nothing to do, appended again and again at the current lengths (or at a start
    that is the tensor of the lengths itself, which the call updates): every row where the oracle puts it."""
    rkv, runner, synth = mods
    n_kv, T, lens = 8, 190, [0, 5, 64, 100, 63, 1]
    counts = [[1, 70, 0, 3, 190, 64], [0, 1, 2, 65, 1, 1], [130, 0, 1, 1, 1, 128], [1, 1, 1, 1, 1, 1]]
    c = synth.alloc_quant_cache([n + 2048 for n in lens], n_kv, torch.device("cuda"))
    ctx = context(rkv, 6, n_kv, n_kv, 64)
    cs, host, g = struct(rkv, c), Host(c, n_kv), gen(8)
    x = [normal(g, 6, T, n_kv, 128).to(torch.bfloat16) for _ in range(2)]
    ctx.quant_store(x[0], x[1], cs, count=i32(lens))
    host.store(x[0], x[1], count=lens)
    for turn in range(6):
        for i, count in enumerate(counts):                 # several calls in flight before the host looks
            k, v = x[i % 2] * (1 + turn), x[1 - i % 2]
            ctx.quant_store(k, v, cs, start=c.len if given == "lengths as start" else None, count=i32(count))
            host.store(k, v, count=count)
        host.check()
    assert ctx.device_status() == 0


# ------------------------------------------------------------------------------------- traces of earlier calls
FORMS = {                     # sequences, positions the context takes, lengths of the healthy call
    "bf16": (1, 20000, [700]),
    "splits": (1, 20000, [700]),
    "cluster": (1, 2048, [130]),
    "balanced": (3, 20000, [900, 300, 64]),
}


def bf16_cache(synth, lens, caps, n_kv, seed):
    c = synth.alloc_cache(caps, lens, n_kv, torch.device("cuda"), fill=0.0)
    for x in (c.k, c.v):
        x.copy_(normal(gen(seed + x.shape[0]), *x.shape).to(torch.bfloat16))
    return c


def reference(c, form, q, n_kv, lens):
    if form != "bf16":
        return quant_reference(Host(c, n_kv), q, n_kv, lens)
    ref = []
    for b, n in enumerate(lens):
        rows = [int(c.row_offset[b]) + h * int(c.cap[b]) for h in range(n_kv)]
        k, v = (np.stack([f64(x[r: r + n]) for r in rows]) for x in (c.k, c.v))
        out, p, _ = O.decode_attention(f64(q[b]), k, v)
        ref.append((out, O.decode_attention(f64(q[b]), k, np.abs(v))[0], p))
    return ref


@pytest.mark.parametrize("form", list(FORMS))
def test_scores_behind_a_pass_with_nan(mods, form):
    """A long pass over a cache with a NaN row far behind, then, on the same context, a healthy one over fewer positions:
    its scores and its selection know nothing of the first."""
    rkv, runner, synth = mods
    n_seq, most, lens = FORMS[form]
    n_kv, group, keep = 2, 4, 50
    ctx = context(rkv, n_seq, n_kv * group, n_kv, most)
    q = normal(gen(7), n_seq, n_kv * group, 128).to(torch.bfloat16)
    out, idx = torch.empty_like(q), torch.empty((n_seq, n_kv, keep), dtype=torch.int32, device="cuda")
    scores = torch.full((n_seq, n_kv, most), -1.0, device="cuda")
    k_small = i32([keep] * n_seq)

    def step(c):
        if form == "bf16":
            ctx.full_attention(q, rkv.cache_struct(c.k, c.v, c.row_offset, c.cap, c.len), out)
            cs = rkv.cache_struct(c.k, c.v, c.row_offset, c.cap, c.len)
        else:
            cs = struct(rkv, c)
            ctx.quant_full_attention(q, cs, out)
        ctx.select_topk(q, cs, k_small, keep, idx, scores=scores)

    long = [most] * n_seq
    if form == "bf16":
        c = bf16_cache(synth, long, long, n_kv, 3)
        c.k[:] = torch.where(torch.arange(c.k.shape[0], device="cuda")[:, None] % most > most // 2, torch.nan, c.k)
    else:
        c = filled(synth, long, n_kv, 3, caps=[(most + 63) // 64 * 64] * n_seq)
        for b in range(n_seq):
            for h in range(n_kv):
                r, cap = head_rows(c, b, h)
                c.k.view(torch.uint8)[r + most // 2: r + most] = 0x7f
    step(c)
    assert ctx.device_status() & rkv.DEV_NONFINITE
    c = bf16_cache(synth, lens, lens, n_kv, 4) if form == "bf16" else filled(synth, lens, n_kv, 4)
    scores.fill_(-1.0)
    step(c)
    assert ctx.device_status() == 0
    ref = reference(c, form, q, n_kv, lens)
    for b, n in enumerate(lens):
        check_scores(scores[b], ref[b][2], group, f"sequence {b}")
        assert (scores[b, :, n:] == -1).all()
        want = ref[b][2].reshape(n_kv, group, -1).max(axis=1)
        for h in range(n_kv):
            why = O.check_topk_set(want[h], min(keep, n), idx[b, h, : min(keep, n)].cpu().numpy())
            assert why is None, why


@pytest.mark.parametrize("bad", ["cap", "offset", "outside"])
@pytest.mark.parametrize("form", ["splits", "cluster", "cluster batch", "balanced"])
def test_second_half_of_a_bad_layout(mods, form, bad):
    """A sequence whose layout does not suit the blocks is left alone by the scores and by the record of its query, and
    none of its positions is selected, although the workspace still holds a healthy pass over it."""
    rkv, runner, synth = mods
    n_seq, most = {"splits": (1, 20000), "cluster": (1, 2048), "cluster batch": (3, 2048), "balanced": (3, 20000)}[form]
    n_kv, group, keep, lens, b = 2, 4, 50, [1900, 300, 700][:n_seq], n_seq // 2
    c = filled(synth, lens, n_kv, 9)
    ctx = context(rkv, n_seq, n_kv * group, n_kv, most)
    q = normal(gen(7), n_seq, n_kv * group, 128).to(torch.bfloat16)
    ref = quant_reference(Host(c, n_kv), q, n_kv, lens)
    cs, k_small = struct(rkv, c), i32([keep] * n_seq)

    def buffers():
        return (torch.full_like(q, 7.0), torch.full((n_seq, n_kv, keep), -2, dtype=torch.int32, device="cuda"),
                torch.full((n_seq, n_kv, most), -1.0, device="cuda"), torch.full_like(q, 5.0))

    def in_one_call(out, idx, scores, last):
        ctx.quant_full_step(q, cs, k_small, keep, out, idx, scores=scores, q_last_full=last)

    def in_halves(out, idx, scores, last):
        ctx.quant_full_attention(q, cs, out)
        ctx.select_topk(q, cs, k_small, keep, idx, scores=scores, q_last_full=last)

    def in_three(out, idx, scores, last):
        ctx.quant_full_attention(q, cs, out)
        ctx.score_keys(q, cs, k_small, keep, scores=scores, q_last_full=last)
        ctx.select_topk(None, cs, k_small, keep, idx)

    for call in (in_one_call, in_halves, in_three):
        call(*buffers())                                    # every sequence in order: logits and statistics of all
        assert ctx.device_status() == 0
        t = {"cap": c.cap, "offset": c.row_offset, "outside": c.row_offset}[bad]
        kept = int(t[b])
        t[b] = {"cap": kept + 32, "offset": kept + 32, "outside": c.n_rows}[bad]
        out, idx, scores, last = buffers()
        call(out, idx, scores, last)
        assert ctx.device_status() == rkv.DEV_BAD_LAYOUT
        t[b] = kept
        for i, n in enumerate(lens):
            if i == b:
                assert (out[i] == 0).all() and (idx[i] == -1).all() and (scores[i] == -1).all() and (last[i] == 5).all()
                continue
            check_out(out[i], ref[i], f"sequence {i}")
            check_scores(scores[i], ref[i][2], group, f"sequence {i}")
            assert torch.equal(last[i], q[i])
            want = ref[i][2].reshape(n_kv, group, -1).max(axis=1)
            for h in range(n_kv):
                why = O.check_topk_set(want[h], keep, idx[i, h].cpu().numpy())
                assert why is None, why


# -------------------------------------------------------------------------------------------------------------- rebuild
@pytest.mark.parametrize("bad", ["before", "behind", "last head", "capacity"])
def test_rebuild_leaves_rows_outside_the_small_cache_alone(mods, bad):
    """A small cache whose sequence does not lie inside its buffers: flagged, nothing of that sequence is written."""
    rkv, runner, synth = mods
    n_kv, keep, b = 2, 20, 1
    c = filled(synth, [200, 300], n_kv, 5)
    small = synth.alloc_cache([32, 32], [7, 7], n_kv, torch.device("cuda"), fill=5.0)
    whole = small.k                                        # 128 rows, of which the struct says fewer where rows are cut
    ctx = context(rkv, 2, n_kv, n_kv, 512, keep)
    rows = 128 if bad in ("before", "capacity") else 127
    if bad == "before":
        small.row_offset[b] = -32
    elif bad == "behind":
        small.row_offset[b] = 65
    elif bad == "capacity":
        small.cap[b] = 33
    sc = rkv.cache_struct(small.k[:rows], small.v[:rows], small.row_offset, small.cap, small.len)
    idx = torch.arange(keep, dtype=torch.int32, device="cuda").repeat(2, n_kv, 1).contiguous()
    ctx.quant_gather_small(idx, i32([keep, keep]), keep, struct(rkv, c), sc)
    assert ctx.device_status() == rkv.DEV_BAD_LAYOUT
    assert small.len.tolist() == [keep, 7] and (whole[64:] == 5).all() and (small.v[64:] == 5).all()
    host = Host(c, n_kv)
    for h in range(n_kv):
        want = torch.from_numpy(host.values("k", 0, h, 200)[:keep]).float().to(torch.bfloat16)
        assert torch.equal(whole[32 * h: 32 * h + keep].cpu(), want)


# ------------------------------------------------------------------------------------------------------------- rotation
def test_attention_right_behind_a_rotation_into_the_cache(mods):
    """With one KV head, rkv_rope's keys and values can be the rows of a bf16 cache themselves.  The attention behind it
    may request its first tiles ahead only of launches that leave the cache alone, which this one does not."""
    rkv, runner, synth = mods
    n, group = 4096, 4
    c = synth.alloc_cache([n], [n], 1, torch.device("cuda"), fill=0.0)
    cs = rkv.cache_struct(c.k, c.v, c.row_offset, c.cap, c.len)
    ctx = context(rkv, 1, group, 1, n)
    g, pos, table = gen(3), torch.arange(n, dtype=torch.int32, device="cuda"), rkv.RopeTable(device="cuda")
    q = torch.empty((n, group, 128), dtype=torch.bfloat16, device="cuda")
    qkv = [(normal(g, n, (group + 2) * 128) * s).to(torch.bfloat16) for s in (1.0, 2.0, 0.5)]

    def run(x, wait):
        ctx.rope(x, pos, table, q, c.k.view(n, 1, 128), c.v.view(n, 1, 128))
        if wait:
            torch.cuda.synchronize()
        out = torch.empty((1, group, 128), dtype=torch.bfloat16, device="cuda")
        ctx.full_attention(q[-1:], cs, out)
        return out

    want = [run(x, True) for x in qkv]
    got = [run(x, False) for _ in range(20) for x in qkv]
    for i, out in enumerate(got):
        assert torch.equal(out, want[i % 3])
    assert ctx.device_status() == 0


# -------------------------------------------------------------------------------------------------------- other calls
@pytest.mark.parametrize("order", ["tokens first", "one row for all", "batch of one"])
def test_store_rows_in_other_orders(mods, order):
    """Sequences that lie closer than tokens do, a batch that repeats one sequence's rows, strides that are never taken."""
    rkv, runner, synth = mods
    n_kv, T, g = 3, 100, gen(17)
    B = 1 if order == "batch of one" else 3
    if order == "tokens first":
        k, v = (normal(g, T, B, n_kv, 128).to(torch.bfloat16).transpose(0, 1) for _ in range(2))
        assert k.stride(0) < k.stride(1)
    elif order == "one row for all":
        k, v = (normal(g, 1, T, n_kv, 128).to(torch.bfloat16).expand(B, T, n_kv, 128) for _ in range(2))
    else:
        wide = normal(g, T, 2, n_kv, 128).to(torch.bfloat16)
        k, v = (wide[None, :, i].as_strided((1, T, n_kv, 128), (7, 2 * n_kv * 128, 128, 1), i * n_kv * 128) for i in range(2))
    c = synth.alloc_quant_cache([200] * B, n_kv, torch.device("cuda"))
    ctx, host = context(rkv, B, n_kv, n_kv, 256), Host(c, n_kv)
    for count in ([T, 63, 1][:B], [5, 37, T][:B]):
        ctx.quant_store(k, v, struct(rkv, c), count=i32(count))
        host.store(k, v, count=count)
        host.check()
    assert ctx.device_status() == 0


def test_balanced_pass_captured_and_replayed(mods):
    """Two graphs of a full step over a batch in the balanced form, on one workspace, replayed in turn while the lengths
    grow and shrink on the device: each replay as the eager call on a context of its own."""
    rkv, runner, synth = mods
    n_kv, group, keep, most = 2, 4, 100, 9000
    lens = [[9000, 1, 3000], [128, 0, 8999], [6000, 6000, 6000], [1, 1, 129]]
    side = torch.cuda.Stream()
    shared, own = (context(rkv, 3, n_kv * group, n_kv, most, 128) for _ in range(2))
    k_small, steps = i32([keep] * 3), []
    for seed in (1, 2):
        c = filled(synth, [most] * 3, n_kv, seed)
        q = normal(gen(seed), 3, n_kv * group, 128).to(torch.bfloat16)

        def buffers():
            return (torch.zeros_like(q), torch.zeros((3, n_kv, 128), dtype=torch.int32, device="cuda"),
                    torch.zeros((3, n_kv, most), device="cuda"))

        def step(ctx, t, q=q, cs=struct(rkv, c)):
            ctx.quant_full_attention(q, cs, t[0])
            ctx.score_keys(q, cs, k_small, 128, scores=t[2])
            ctx.select_topk(None, cs, k_small, 128, t[1])

        kept, eager = buffers(), buffers()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            step(shared, kept)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step(shared, kept)
        step(own, eager)               # (the same calls on both sides: scores past a length stay what an earlier call wrote)
        torch.cuda.synchronize()
        steps.append((c, step, graph, kept, eager))
    for ns in lens + lens[::-1]:
        for c, step, graph, kept, eager in steps:
            c.len.copy_(i32(ns))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _, _, graph, _, _ in steps:
                graph.replay()
        for _, step, _, _, eager in steps:
            step(own, eager)
        torch.cuda.synchronize()
        for _, _, _, kept, eager in steps:
            for a, b in zip(kept, eager):
                assert torch.equal(a, b)
    assert shared.device_status() == 0 and own.device_status() == 0


@pytest.mark.parametrize("left_by", ["8 bits", "bf16"])
@pytest.mark.parametrize("captured", ["the step", "the scores"])
def test_selection_behind_scores_that_were_never_selected(mods, left_by, captured):
    """A score pass without its selection leaves its keys' histogram in the workspace.  A full step of the bf16 cache
    behind it selects as ever, also where one of the two is a graph, so that the host cannot know what runs before what."""
    rkv, runner, synth = mods
    n_kv, group, n, keep = 2, 4, 3000, 200
    ctx = context(rkv, 1, n_kv * group, n_kv, n, keep)
    b = bf16_cache(synth, [n], [n], n_kv, 5)
    bs = rkv.cache_struct(b.k, b.v, b.row_offset, b.cap, b.len)
    c = filled(synth, [n], n_kv, 6)
    cs, k_small = struct(rkv, c), i32([keep])
    q = normal(gen(7), 1, n_kv * group, 128).to(torch.bfloat16)
    other = torch.empty_like(q)
    out, idx = torch.empty_like(q), torch.empty((1, n_kv, keep), dtype=torch.int32, device="cuda")

    def step():
        ctx.full_step(q, bs, k_small, keep, out, idx)

    def scores():
        if left_by == "bf16":
            ctx.full_attention(q, bs, other)
            ctx.score_keys(q, bs, k_small, keep)
        else:
            ctx.quant_full_attention(q, cs, other)
            ctx.score_keys(q, cs, k_small, keep)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.current_stream())
        step()
        want = (out.clone(), idx.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step() if captured == "the step" else scores()
        step()                                    # (behind a captured score pass, which has not run)
        for _ in range(3):
            idx.fill_(-2)
            out.zero_()
            if captured == "the step":
                scores()
                graph.replay()
            else:
                graph.replay()
                step()
            side.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(idx, want[1])
    assert ctx.device_status() == 0
