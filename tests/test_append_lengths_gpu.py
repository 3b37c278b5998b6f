"""bf16 appends inside attention launches, many in flight: the lengths grow by one per call, every row lands behind the last,
and every call attends over exactly the rows up to its own (64-position tiles are crossed on the way)."""
import numpy as np
import pytest
import torch

from oracle import rkv_oracle as O
from test_quant_gpu import context, f64, gen, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2411_05787_b200 import rkv, synth
    return rkv, synth


@pytest.mark.parametrize("form", ["streaming", "cluster", "cluster and full cache"])
@pytest.mark.parametrize("lens", [[0], [62, 0, 127], [511]])
def test_appended_rows_and_lengths(mods, form, lens):
    rkv, synth = mods
    n_kv, group, steps, B = 2, 4, 70, len(lens)
    dev = torch.device("cuda")
    most = max(lens) + steps
    ctx = context(rkv, B, n_kv * group, n_kv, most, most)
    made = [synth.alloc_cache([most] * B, lens, n_kv, dev, fill=0.0) for _ in range(2)]
    g = gen(sum(lens) + 1)
    for c in made:
        for x in (c.k, c.v):
            x.copy_(normal(g, *x.shape).to(torch.bfloat16))
    (small, full), (ss, fs) = made, [rkv.cache_struct(c.k, c.v, c.row_offset, c.cap, c.len) for c in made]
    q = normal(g, steps, B, n_kv * group, 128).to(torch.bfloat16)
    k, v = (normal(g, steps, B, n_kv, 128).to(torch.bfloat16) for _ in range(2))
    out = torch.empty_like(q)
    for t in range(steps):
        if form == "streaming":
            ctx.append_full_attention(q[t], k[t], v[t], ss, out[t])
        else:
            ctx.append_small_step(q[t], k[t], v[t], fs if form.endswith("full cache") else None, ss, out[t])
    assert ctx.device_status() == 0
    grown = [small] + ([full] if form.endswith("full cache") else [])
    for c in grown:
        assert c.len.tolist() == [n + steps for n in lens]
        for b, n in enumerate(lens):
            for h in range(n_kv):
                at = int(c.row_offset[b]) + h * most + n
                assert torch.equal(c.k[at: at + steps], k[:, b, h]) and torch.equal(c.v[at: at + steps], v[:, b, h])
    for t in (0, 1, 2, steps // 2, steps - 1):
        for b, n in enumerate(lens):
            rows = [slice(int(small.row_offset[b]) + h * most, int(small.row_offset[b]) + h * most + n + t + 1) for h in range(n_kv)]
            kk, vv = (np.stack([f64(x[r]) for r in rows]) for x in (small.k, small.v))
            want = O.decode_attention(f64(q[t, b]), kk, vv)[0]
            mass = O.decode_attention(f64(q[t, b]), kk, np.abs(vv))[0]
            # p goes through bf16 (2^-8 of S), the output as well, the rest is fp32 noise: twice the former
            assert (np.abs(f64(out[t, b]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * mass).all()
