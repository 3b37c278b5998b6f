"""Results of the paged cache's calls that are known to the last bit."""
import pytest
import torch

from test_paged_gpu import Pool, i32, normal, gen, rkv  # noqa: F401  (rkv: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout,rot,scaling,factor", [("half", 128, "none", 1.0), ("interleaved", 128, "bands", 8.0),
                                                       ("half", 48, "ramp", 4.0), ("interleaved", 64, "linear", 2.0)])
@pytest.mark.parametrize("T", [1, 4, 5, 700])
def test_appended_rows_are_those_that_rope_turns(rkv, T, layout, rot, scaling, factor, dtype):
    """Tokens, chunks and prompts, near and far: one angle, one sine and cosine, one product."""
    n_q, n_kv, page, starts = 14, 2, 128 if T > 4 else 32, [0, 7, 70001]
    pool = Pool(rkv, [s + T for s in starts], n_kv, page, T, lens=starts)
    ctx = rkv.Context(len(starts), n_q, n_kv, 1024, 64)
    x = normal(gen(rot + T), len(starts), T, (n_q + 2 * n_kv) * 128).to(dtype)
    q = torch.empty((len(starts), T, n_q, 128), dtype=torch.bfloat16, device="cuda")
    table = rkv.RopeTable(rot, 500000.0, layout, scaling, factor)
    ctx.paged_append(x, pool.struct(), table, q)
    for b, s in enumerate(starts):
        want = [torch.empty((T, h, 128), dtype=torch.bfloat16, device="cuda") for h in (n_q, n_kv, n_kv)]
        ctx.rope(x[b], i32(list(range(s, s + T))), table, *want)
        at = torch.arange(s, s + T, device="cuda")
        pages, rows = pool.table[b].long()[at // page], at % page
        assert torch.equal(q[b], want[0])
        assert torch.equal(pool.k[pages, :, rows], want[1]) and torch.equal(pool.v[pages, :, rows], want[2])
    assert ctx.device_status() == 0


@pytest.mark.parametrize("B", [16, 40])
def test_what_all_values_have_in_common_comes_through_behind_a_prefix(rkv, B):
    """All values alike: out = sum p v / sum p is that value as long as both sums are of the same p; 64 and 160 rows of a head
    (one block of 128 rows, and two).  A row's largest probability is 2^s beside a maximum of an earlier tile (0 < s < 8), so
    it is rounded for the products, by up to 2^-8 of it; 1.9921875 has half a bf16 step of 2^-9 of it.  The sums of
    products that are exact in fp32 (bf16 x bf16) are off by far less than that, so the output has to be that value itself."""
    n_q, n_kv, page, v = 8, 2, 64, 1.9921875
    n_cta = min(torch.cuda.get_device_properties(0).multi_processor_count // n_kv, 64)      # CTAs that share the prefix
    tiles = 2 * n_cta + 1
    prefix = tiles * 64
    pool = Pool(rkv, [prefix] * B, n_kv, page, 4, lens=[prefix] * B, bounds=False, shared=tiles)
    pool.v.fill_(v)
    pool.k.zero_()
    pool.k[..., 0] = -256.0                       # scores far below the two that count
    at = pool.shared.long()
    pool.k[at[0], :, 5, 0] = 0.0                  # the first tile of the first CTA: the maximum that its rows keep
    pool.k[at[2 * n_cta], :, 9, 0] = 8.0          # its third tile (the same group of warps whatever the form)
    q = torch.zeros((B, n_q, 128), dtype=torch.bfloat16, device="cuda")
    x = torch.linspace(1.0, 7.6, B * n_q, device="cuda").view(B, n_q)      # s = x 8 log2(e) / sqrt(128) = 1.02 x
    q[..., 0] = x.to(torch.bfloat16)
    ctx = rkv.Context(B, n_q, n_kv, prefix, 64)
    ctx.set_option(rkv.OPT_SHARED_MIN, 0)
    out, before = torch.empty_like(q), ctx.launch_count
    ctx.paged_attention(q, pool.struct(), out, shared=pool.shared)
    assert ctx.device_status() == 0 and ctx.launch_count - before == 3
    assert (out == v).all(), f"{int((out != v).any(-1).sum())} of {B * n_q} rows differ"
