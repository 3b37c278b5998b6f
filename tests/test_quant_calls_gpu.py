"""The 8-bit cache's calls where they meet other calls: lengths read while they are about to change, workspaces that an
earlier call has left its traces in, sequences that one call refuses and the next one reads."""
import pytest
import torch

from test_quant_gpu import Host, context, gen, i32, normal, struct

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
