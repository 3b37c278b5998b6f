"""The halves of a decode token over paged caches, without a GPU: the append is part of the attention half, as it is for
the other caches, so that a token without its decoder still does all that the cache costs."""
import pytest

from test_quant_cpu import built  # noqa: F401  (the libraries are there)

pytestmark = pytest.mark.usefixtures("built")


class _Tensor:
    def view(self, *shape):
        return self

    def __getitem__(self, i):
        return self


class _State:
    def __init__(self, calls):
        self.calls, self.out, self.full = calls, _Tensor(), _Tensor()
        self.full.len = None

    def append(self, *args, **kwargs):
        self.calls.append("append")

    def attend(self, *args, **kwargs):
        self.calls.append("attend")
        return self.out

    def attend_selected(self, *args, **kwargs):
        self.calls.append("attend_selected")
        return self.out


@pytest.mark.parametrize("kind,attends", [("small", "attend_selected"), ("check", "attend_selected"), ("full", "attend")])
@pytest.mark.parametrize("with_harness,with_attention", [(True, True), (False, True), (True, False)])
def test_halves_of_a_token(monkeypatch, kind, attends, with_harness, with_attention):
    from paper_2411_05787_b200 import harness as H
    calls = []
    for name in ("embed", "gemv", "gemv_swiglu", "argmax"):
        monkeypatch.setattr(H, name, lambda *args, **kwargs: calls.append("harness"))
    dec = object.__new__(H.LlamaDecoder)
    dec.s, dec.page, dec.capture, dec.table, dec.full_hint = H.LlamaShape(n_layers=2), 16, None, None, 64
    dec.layers_w = [dict.fromkeys(("wqkv", "wo", "wgu", "wd", "norm1", "norm2"))] * 2
    dec.states = [_State(calls) for _ in range(2)]
    for name in ("x", "qkv", "act", "logits", "token", "embed_w", "lm_head", "final_norm"):
        setattr(dec, name, _Tensor())
    dec.q = dec.k = dec.v = [_Tensor(), _Tensor()]
    dec.token_step(kind, with_harness=with_harness, with_attention=with_attention)
    assert [c for c in calls if c != "harness"] == ["append", attends] * 2 * with_attention
    assert ("harness" in calls) == with_harness
