"""What is refused of a predictor with a norm (no GPU): see test_layers_cpu on contexts and addresses that are none."""
import ctypes as C

import pytest
import torch

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


def _host_context():
    """A context that was never created, whose device is the host."""
    from paper_2303_13803_amd import Context
    c = object.__new__(Context)
    c.device = -1
    return c


def _params(F=5, H=64):
    sizes = {"W1": (H, 2 * F), "b1": (H,), "W2": (H, H), "b2": (H,), "W3": (H,), "b3": (1,), "W1sm": (H,), "W3slow": (H,), "b3slow": (1,), "ln_w": (2 * F,), "ln_b": (2 * F,)}
    return {k: torch.zeros(v) for k, v in sizes.items()}


def test_a_predictor_of_parameters_of_its_sizes():
    params = _params()
    p = _host_context().predictor(params, 2.0, mem_feature=3, mem_limit=0.5, sm=(1, 2), slow_limit=0.25, norm_eps=1e-3)
    assert (p.F, p.H, p.scale, p.mem_feature, p.mem_limit, p.sm_on_feature, p.sm_off_feature, p.slow_limit) == (5, 64, 2.0, 3, 0.5, 1, 2, 0.25)
    assert p.ln_eps == C.c_float(1e-3).value and p.d_W1 == params["W1"].data_ptr() and p.d_ln_b == params["ln_b"].data_ptr() and p.d_b3_slow == params["b3slow"].data_ptr()
    plain = _host_context().predictor({k: params[k] for k in ("W1", "b1", "W2", "b2", "W3", "b3")}, 1.0)
    assert plain.d_W1sm is None and plain.d_W3_slow is None and plain.d_b3_slow is None and plain.d_ln_w is None and plain.d_ln_b is None and plain.ln_eps == 0.0


@pytest.mark.parametrize("name", ["ln_w", "ln_b", "W1sm", "W3slow", "b3slow", "W2", "b2", "W3", "b3"])
def test_parameters_of_other_sizes(name):
    """A norm's weight made for F features instead of 2 F would be read past its end."""
    params = _params()
    params[name] = params[name][: params[name].shape[0] // 2]
    with pytest.raises(ValueError, match=name):
        _host_context().predictor(params, 1.0, sm=(1, 2), slow_limit=0.5, norm_eps=1e-5)


@pytest.mark.parametrize("change", [{"ln_w": torch.zeros(10, dtype=torch.float64)}, {"ln_b": torch.zeros(20)[::2]}, {"W1": torch.zeros(10, 64).t()}, {"b2": None}])
def test_parameters_of_other_kinds_and_places(change):
    with pytest.raises(TypeError):
        _host_context().predictor({**_params(), **change}, 1.0, sm=(1, 2), slow_limit=0.5, norm_eps=1e-5)


def test_numbers_that_lose_their_upper_bits_on_the_way():
    """2^32 + 5 workloads are not five, and layer 2^32 + 1 is not layer 1."""
    from paper_2303_13803_amd import MuxmatchError
    c = _host_context()
    with pytest.raises(ValueError, match="x_on"):
        c._side(torch.empty((2 ** 32 + 5, 1), device="meta"), 1, "x_on")
    x = torch.zeros(3, 8)
    for layer in (2 ** 32 + 1, -1, 65536):
        with pytest.raises(MuxmatchError, match="layer"):
            c.dropout(x, x, 0.5, 1, layer=layer)
