"""The decode loop over paged caches: every append and attention call of two layers against the oracle (tolerances of the
bf16 loop's test for the outputs; keys and values within half a bf16 step and 2^-14 of the projection's rows)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from oracle import quant_oracle as QO

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2411_05787_b200 import harness
    return harness


def f64(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("page,scaling", [(16, None), (64, dict(scaling="bands", factor=8.0, trained_len=512))])
def test_decode_loop_over_paged_caches(H, page, scaling):
    shape = H.LlamaShape(hidden=512, n_layers=3, n_q=4, n_kv=2, ffn=1024, vocab=1000)
    dec = H.LlamaDecoder(shape, prompt_len=1500, max_new=24, k_small=128, qc_stride=4, threshold=0.9, seed=11, page=page,
                         top_pages=6, rope_scaling=scaling)
    g = torch.Generator(device="cpu"); g.manual_seed(12)
    dec.prefill(torch.randint(0, shape.vocab, (1500,), generator=g).to("cuda"))
    assert all(int(st.full.len[0]) == 1500 for st in dec.states)
    kw = dict(scaling or {})
    f, amp = QO.rope_frequencies(128, shape.theta, **kw)
    records = []
    dec.capture = ({0, 2}, records)
    for t in range(1, 13):
        dec.token_step("full" if t % 4 == 0 else dec.kind_of(t))
    torch.cuda.synchronize()
    assert dec.ctx.device_status() == 0 and len(records) == 24
    for r in records:
        st, n = dec.states[r["layer"]], r["len"]
        row = st.full.table[0].tolist()
        k, v = (PO.rows(f64(x), row, page, n) for x in (st.full.k, st.full.v))
        x = f64(r["qkv"]).reshape(1, 8, 128)
        for got, want in ((k[:, -1], QO.rope(x[:, 4:6], [n - 1], f, amp, "half")[0]), (v[:, -1], x[0, 6:])):
            assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -14).all()
        q, at = f64(r["q"][0]), None
        if r["kind"] != "full":
            at = []
            for h in range(2):
                held = [k[h, i: i + page] for i in range(0, n, page)]
                s = PO.scores(q[2 * h: 2 * h + 2], np.array([p.min(0) for p in held]), np.array([p.max(0) for p in held]))
                want = PO.select(s, 6, 1, 1)
                assert r["pages"][0, h].tolist() == want
                at.append([p for i in want for p in range(i * page, min((i + 1) * page, n))])
        want, _ = PO.attend(q, k, v, at=at)
        got = f64(r["out"][0])
        assert np.abs(got - want).max() <= 2e-2
        assert np.linalg.norm(got - want) <= 5e-3 * max(np.linalg.norm(want), 1e-30), (r["layer"], r["kind"])
    dec.capture = None
    side = torch.cuda.Stream()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(gr, stream=side):
            dec.token_step("small")
            dec.token_step("full")
    gr.replay(); gr.replay()
    torch.cuda.synchronize()
    assert all(int(st.full.len[0]) == 1516 for st in dec.states) and dec.ctx.device_status() == 0


def test_paged_caches_hold_bf16(H):
    with pytest.raises(ValueError):
        H.LlamaDecoder(H.LlamaShape(hidden=512, n_layers=1, n_q=4, n_kv=2, ffn=1024, vocab=1000), 16, 4, 8, 4, 0.9, cache_bits=8,
                       page=16)
