"""GPU: samples and workloads that stand out do not change what is said of the others."""
import numpy as np
import pytest
import torch

import fit_close as close
import fit_reference as ref
from gpu_util import dev
from test_gpu_fit import SM, call, definition, predictor, problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2303_13803_amd as mm
    c = mm.Context(64, 64)
    yield c
    c.close()


def same_bits(a, b, names):
    for name in names:
        assert (a[name].view(np.int32) == b[name].view(np.int32)).all(), name


def predictions(ctx, s):
    out = [torch.full((len(s["on"]),), 7.0, device="cuda") for _ in range(2 if s["target_slow"] is not None else 1)]
    ctx.predict_pairs(predictor(ctx, s), dev(s["x_on"]), dev(s["x_off"]), dev(s["on"]), dev(s["off"]), *out)
    return dict(zip(("sigma", "sigma_slow"), (o.cpu().numpy() for o in out)))


# ---- targets of samples that name no pair

@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("F", [16, 70])
@pytest.mark.parametrize("count", [30, 20000])
@pytest.mark.parametrize("fill", [1e9, -1e20, 3e38, np.inf])
def test_targets_of_samples_that_name_no_pair(ctx, fill, count, F, H):
    """In the same 32 samples as real ones, and in others: every bit is what it is with targets like all others there."""
    s = problem(70, count, F, H, slow=True, missing=True)
    none = (s["on"] < 0) | (s["off"] >= 40)
    assert none.any() and not none.all()
    s["target"][none], s["target_slow"][none] = 0.5, 0.5
    plain = call(ctx, s, (0.1, 2, 3))
    s["target"][none], s["target_slow"][none] = fill, fill
    filled = call(ctx, s, (0.1, 2, 3))
    same_bits(plain, filled, plain)
    s = close.away_from_kinks(s, (0.1, 2, 3))
    close.check(call(ctx, s, (0.1, 2, 3)), close.room(s, (0.1, 2, 3), longest=count / 64))


# ---- an SM feature that is no fraction.  Workload 7 and workload 9 have it, so that only a pair of both has a share of that size:
# min(1 + v, v); beside others either's share is an ordinary one.

def with_large_shares(seed, count, H, value, F=16, **kw):
    s = problem(seed, count, F, H, norm=True, sm=True, slow=True, **kw)
    s["x_on"][7, SM[0]], s["x_off"][9, SM[1]] = -value, value
    both = (s["on"] == 7) & (s["off"] == 9)
    s["on"][both] = 8
    return s


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("count", [1000, 5003, 20001])
@pytest.mark.parametrize("value", [5e3, 1e9, 1e12, 1e18])
@pytest.mark.parametrize("named", [False, True])
def test_predictions_beside_a_large_sm_share(ctx, named, value, count, H):
    """As few pairs are predicted and as many are; 1e-5 of every prediction, and of the pair with that share what its own sums may be off.  (Squares of
    features beyond 1.8e19 pass the largest float32, 3.4e38, and with them that row's variance.)"""
    s = with_large_shares(71, count, H, value)
    if named:
        s["on"][17], s["off"][17] = 7, 9
    with np.errstate(over="ignore"):
        expected = definition(s)
    got = predictions(ctx, s)
    others = np.arange(count) != (17 if named else -1)
    for name in got:
        value64, bound = expected[name]
        assert (np.abs(got[name] - value64)[others] <= 1e-5 * value64[others]).all(), name
        ref.within(got[name][~others], value64[~others], bound[~others], name)


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("count, n", [(40, 50), (20001, 50), (40, 500)])
@pytest.mark.parametrize("value", [4e3, 1e9, 1e12])
@pytest.mark.parametrize("which", ["unnamed", "half named", "named"])
def test_a_fit_beside_a_large_sm_share(ctx, which, value, count, n, H):
    """"half named": by samples that name no pair, as their other index is out of range."""
    s = with_large_shares(72, count, H, value, n=n, missing=True)
    if which == "half named":
        s["on"][:2], s["off"][:2] = (7, -1), (-3, 9)
    if which == "named":
        s["on"][5], s["off"][5] = 7, 9
    with np.errstate(over="ignore"):
        s = close.away_from_kinks(s, (0.1, 2, 3))
        assert which != "named" or s["on"][5] == 7
        expected = close.room(s, (0.1, 2, 3), longest=count / 64)
        close.check(call(ctx, s, (0.1, 2, 3)), expected)
    alone = call(ctx, s, (0.1, 2, 3), want=False)
    close.check(alone, {k: expected[k] for k in alone})


# ---- features that are not there, of samples whose targets are not there either

@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("F", [16, 40, 100])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("large", [False, True])
def test_features_nobody_has_measured(ctx, large, value, norm, F, H):
    """A workload without metrics, in pairs nobody has measured: the loss and gradients are those without these samples to the bit; their
    predictions are NaN.  large: also through float32 products, where there is no norm."""
    s = problem(73, 700, F, H, norm=norm, sm=True, slow=True, missing=True)
    if large:
        s["x_off"][3, 4] = 1e5
        s["params"]["W1"][:, F + 4] /= np.float32(1e5)
    s["x_on"][7] = value
    s["x_off"][9, 2:] = value
    blank = ((s["on"] == 7) | (s["off"] == 9)) & (s["on"] >= 0) & (s["off"] < 40)
    assert blank.any()
    s["target"][blank], s["target_slow"][blank] = np.nan, np.nan
    got = call(ctx, s, (0.1, 2, 3))
    without = call(ctx, dict(s, on=np.where(blank, -1, s["on"]).astype(np.int32)), (0.1, 2, 3))
    assert np.isnan(got["sigma"][blank]).all() and np.isnan(got["sigma_slow"][blank]).all()
    assert (got["sigma"][~blank] == without["sigma"][~blank]).all()
    same_bits(got, without, [k for k in got if not k.startswith("sigma")])
    assert all(np.isfinite(got[k]).all() for k in s["params"])


@pytest.mark.parametrize("F", [16, 100])
@pytest.mark.parametrize("norm", [False, True])
def test_features_that_are_not_finite_show_where_something_was_measured(ctx, norm, F):
    s = problem(74, 300, F, 64, norm=norm)
    s["x_on"][7] = np.nan
    assert (s["on"] == 7).any()
    got = call(ctx, s)
    assert np.isnan(got["loss"]).all() and all(np.isnan(got[k]).any() for k in ("W3", "b3", "W2", "b2", "W1", "b1"))


# ---- weights of any size

@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("size", [1e25, 1e32, 1e36])
@pytest.mark.parametrize("which", ["W1", "W2"])
def test_predictions_with_weights_of_any_size(ctx, which, size, H):
    """Predictions are then certain; they are what they are by themselves, where few pairs are asked for."""
    s = problem(75, 5000, 16, H)
    s["params"][which] *= np.float32(size)
    if which == "W1":
        s["params"]["W2"] *= np.float32(1e-30)
    with np.errstate(over="ignore"):
        value, bound = definition(s)["sigma"]
    got = predictions(ctx, s)["sigma"]
    few = np.concatenate([predictions(ctx, dict(s, on=s["on"][k:k + 1000], off=s["off"][k:k + 1000]))["sigma"] for k in range(0, 5000, 1000)])
    # (exp(-z) beyond 2^128 is an infinity, and the prediction 0 where it is below 2^-128)
    ref.within(few, value, bound + 2.0 ** -128, "few")
    ref.within(got, value, bound + 2.0 ** -128, "many")


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("w2, w3", [(1e-13, 1e-20), (1e-20, 1e-12), (1e-6, 1e-22)])
def test_gradients_through_weights_of_next_to_nothing(ctx, w2, w3, H):
    """Their products are far above the smallest numbers there are, also where scales to fp16's range would not be."""
    s = problem(76, 300, 16, H)
    s["params"]["W2"] *= np.float32(w2)
    s["params"]["W3"] *= np.float32(w3)
    s = close.away_from_kinks(s, margin=0.0)
    got, expected = call(ctx, s, None, 1.0), close.room(s, None, 1.0, longest=10)
    # (the second layer's bias decides which of its units are open)
    close.check(got, {k: expected[k] for k in ("W1", "b1", "W2", "b2", "ln_w", "ln_b")})


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("norm, sm", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("bias", [-1e9, -1e20, -3e38])
def test_units_closed_by_their_bias(ctx, bias, norm, sm, H):
    """However far: the others' values are scaled by what units can pass on, not by what closes some."""
    s = problem(77, 5000, 16, H, norm=norm, sm=sm)
    s["params"]["b1"][[3, 40]] = bias
    s = close.away_from_kinks(s, (0.1, 2, 3))
    expected = close.room(s, (0.1, 2, 3), longest=80)
    got = call(ctx, s, (0.1, 2, 3))
    close.check(got, expected)
    alone = call(ctx, s, (0.1, 2, 3), want=False)
    close.check(alone, {k: expected[k] for k in alone})
    exact = close.evaluate(s)[0]["sigma"]
    assert (np.abs(predictions(ctx, s)["sigma"] - exact) <= 1e-5 * exact).all()
