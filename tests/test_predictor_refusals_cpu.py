"""What is refused of a predictor with a norm (no GPU): see test_layers_cpu on contexts and addresses that are none."""
import ctypes as C

import pytest

from test_layers_cpu import A, _loss, _predictor, ctx, lib  # noqa: F401


@pytest.mark.parametrize("eps, refused", [(2.0 ** -126, False), (2.0 ** -127, True), (1e-45, True), (0.0, True)])
def test_an_eps_below_the_smallest_normal_number(lib, ctx, eps, refused):  # noqa: F811
    """A predictor that is not refused is one whose scratch is not enough."""
    p = _predictor(lib, ln_eps=eps)
    raw = lib.raw_library()
    assert (raw.mf_predictor_loss_work(ctx, C.byref(p), 100) == lib.ERR_ARG) == refused
    assert _loss(lib, ctx, {"ln_eps": eps}, bytes=16) == lib.ERR_ARG
    assert raw.mf_predict_pairs(ctx, C.byref(p), None, 0, None, 0, None, None, 0, None, None) == (lib.ERR_ARG if refused else lib.OK)
    if refused:
        assert raw.mf_score_pairs(ctx, C.byref(p), A, 1, A, 1, A, 4, None) == lib.ERR_ARG
