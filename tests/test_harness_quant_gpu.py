"""The decode loop over 8-bit full caches with scaled rotary positions: every attention call of two layers against the
oracle on the caches' own values (tolerances of the bf16 loop's test)."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as QO
from oracle import rkv_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2411_05787_b200 import harness
    return harness


def f64(t):
    return t.detach().double().cpu().numpy()


def values(cache, n_kv, which, n):
    cap = int(cache.cap[0])
    codes = getattr(cache, which).detach().cpu().view(torch.uint8).numpy().reshape(n_kv, cap, 128)
    scale = f64(getattr(cache, which + "_scale")).reshape(n_kv, cap // 64)
    return np.stack([QO.values(codes[g, :n], scale[g]) for g in range(n_kv)])


def test_decode_loop_over_quant_caches(H):
    shape = H.LlamaShape(hidden=512, n_layers=3, n_q=4, n_kv=2, ffn=1024, vocab=1000)
    dec = H.LlamaDecoder(shape, prompt_len=1500, max_new=24, k_small=128, qc_stride=4, threshold=0.9, seed=11,
                         cache_bits=8, rope_scaling=dict(scaling="bands", factor=8.0, trained_len=512))
    g = torch.Generator(device="cpu"); g.manual_seed(12)
    dec.prefill(torch.randint(0, shape.vocab, (1500,), generator=g).to("cuda"))
    assert all(int(st.full.len[0]) == 1500 and int(st.small.len[0]) == 128 for st in dec.states)
    st0 = dec.states[0]
    idx = st0.topk_idx[0].cpu().numpy()
    small = f64(st0.small.k).reshape(2, -1, 128)
    for h in range(2):           # the small cache holds the selected positions' values, bit for bit
        assert np.array_equal(small[h, :128], values(st0.full, 2, "k", 1500)[h][idx[h, :128]])
    records = []
    dec.capture = ({0, 2}, records)
    for t in range(1, 21):
        n0 = len(records)
        dec.token_step(dec.kind_of(t))
        for r in records[n0:]:   # the row a call appended may raise its block's scale later: look at the cache now
            st = dec.states[r["layer"]]
            r["k"], r["v"] = values(st.full, 2, "k", r["full_len"]), values(st.full, 2, "v", r["full_len"])
    torch.cuda.synchronize()
    assert dec.ctx.device_status() == 0 and len(records) == 40
    assert all(int(st.full.len[0]) == 1520 for st in dec.states)
    refreshed = 0
    for r in records:
        q = f64(r["q"][0])
        if r["kind"] == "check" and int(r["flag"][0]) == 1:
            refreshed += 1
            want, score, _, _ = O.full_step(q, r["k"], r["v"], 128)
            for h in range(2):
                assert O.check_topk_set(score[h], 128, r["topk"][0].cpu().numpy()[h, :128]) is None
        else:
            n = r["small_len"]
            k = f64(r["small_k"]).reshape(2, r["small_cap"], 128)[:, :n]
            v = f64(r["small_v"]).reshape(2, r["small_cap"], 128)[:, :n]
            want, _, _ = O.decode_attention(q, k, v)
        got = f64(r["out"][0])
        assert np.abs(got - want).max() <= 2e-2
        assert np.linalg.norm(got - want) <= 5e-3 * max(np.linalg.norm(want), 1e-30), (r["layer"], r["kind"])
    assert refreshed >= 1
    dec.capture = None
    side = torch.cuda.Stream()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(gr, stream=side):
            dec.token_step("small")
            dec.token_step("full")
    gr.replay(); gr.replay()
    torch.cuda.synchronize()
    assert all(int(st.full.len[0]) == 1524 for st in dec.states) and dec.ctx.device_status() == 0


def test_bits_are_checked(H):
    with pytest.raises(ValueError):
        H.LlamaDecoder(H.LlamaShape(hidden=512, n_layers=1, n_q=4, n_kv=2, ffn=1024, vocab=1000), 16, 4, 8, 4, 0.9, cache_bits=4)
