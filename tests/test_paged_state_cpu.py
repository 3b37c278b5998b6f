"""runner.PagedLayerState is no LayerState: what a paged cache has no counterpart of is refused by name."""
import inspect

import pytest

from test_quant_cpu import built  # noqa: F401  (the libraries are there)

pytestmark = pytest.mark.usefixtures("built")


def test_refreshkv_steps_are_refused_over_pages():
    from paper_2411_05787_b200 import runner
    st = object.__new__(runner.PagedLayerState)
    steps = [n for n, f in vars(runner.LayerState).items() if inspect.isfunction(f) and not n.startswith("_") and n != "append"]
    assert {"refresh", "append_partial", "refresh_select", "check_trigger", "enable_eviction", "refresh_scores_only"} <= set(steps)
    for name in steps:
        with pytest.raises(NotImplementedError, match="paged"):
            getattr(st, name)(None, active=None)
    for name in ("small", "flag", "not_flag", "topk_idx"):
        with pytest.raises(NotImplementedError, match="paged"):
            getattr(st, name)


def test_layers_batched_take_no_paged_states():
    from paper_2411_05787_b200 import runner

    class Out:
        device = "cpu"

    st = object.__new__(runner.PagedLayerState)
    st.out, st.n_seq, st.n_q, st.n_kv = Out, 1, 4, 2
    with pytest.raises(NotImplementedError, match="paged"):
        runner.LayerBatchedSmall([st], 64)
