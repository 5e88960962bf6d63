"""RetentionStep's counts of freed and live slots before there are any, and what reset() leaves (no GPU needed)."""
import pytest
import torch

from test_step_quant_args import step  # noqa: F401


@pytest.mark.parametrize("count", ["n_freed", "n_live"])
def test_nothing_is_listed_before_a_redirect(monkeypatch, request, count):
    """The lists themselves are not written yet: a decode, a store or a return must read none of them."""
    monkeypatch.setattr(torch.utils.deterministic, "fill_uninitialized_memory", True)
    torch.use_deterministic_algorithms(True)             # memory that nobody wrote holds the largest value
    try:
        st = request.getfixturevalue("step")
        assert torch.empty(3, dtype=torch.int32).min() > 0
    finally:
        torch.use_deterministic_algorithms(False)
    assert getattr(st, count).tolist() == [0]


def test_reset_restores_the_maps_and_frees_nothing(step):  # noqa: F811
    maps = step.S.clone()
    assert torch.equal(step.S0, maps) and len(maps) == 60 and step.S.is_contiguous()
    step.S.zero_()
    step.n_freed.fill_(7)
    step.M.fill_(2.0)
    step.reset()
    assert torch.equal(step.S, maps) and torch.equal(step.M, step.M0) and step.n_freed.tolist() == [0]
    step.S0[3] = 41                                      # a caller's own start
    step.reset()
    assert int(step.S[3]) == 41
