"""GPU: gradients as near the definition in float64 as sums in float32 can be expected to be (fit_close), for every kernel's instances, through one
tile of samples and through several; half a product's precision would be seen (test_fit_close_cpu)."""
import pytest
import torch

import fit_close as close
from gpu_util import dev
from test_gpu_fit import call, predictor, problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2303_13803_amd as mm
    c = mm.Context(64, 64)
    yield c
    c.close()


def near(ctx, s, drop, longest):
    s = close.away_from_kinks(s, drop)
    expected = close.room(s, drop, longest=longest)
    close.check(call(ctx, s, drop), expected)
    alone = call(ctx, s, drop, want=False)
    close.check(alone, {k: expected[k] for k in alone})


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("F", [4, 16, 32, 33, 48, 64, 65, 129, 256])
@pytest.mark.parametrize("norm, sm, slow", [(True, True, True), (False, False, False), (False, True, False)])
def test_a_few_samples(ctx, norm, sm, slow, F, H):
    near(ctx, problem(80, 1500, F, H, n=200, m=300, norm=norm, sm=sm, slow=slow), (0.1, 2, 3), 30)


# More than two tiles of samples for some workgroups and two for others: 256 compute units take 32 samples each with 128 units and up
# to 64 features, twice as many with 64 units, and twice that in float32 products.

@pytest.mark.parametrize("F", [8, 32, 48, 64])
@pytest.mark.parametrize("norm, extra", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("H, count", [(64, 40003), (64, 33000), (128, 20011), (128, 16500)])
def test_several_tiles_a_workgroup(ctx, H, count, norm, extra, F):
    near(ctx, problem(81, count, F, H, n=500, m=400, norm=norm, sm=extra, slow=extra, missing=True), (0.1, 2, 3), count / 64)


@pytest.mark.parametrize("F, norm", [(65, True), (130, True), (200, False), (20, False), (40, False)])
@pytest.mark.parametrize("H, count", [(64, 70001), (128, 40003)])
def test_several_tiles_a_workgroup_in_float32_products(ctx, H, count, F, norm):
    """Of many features, and without a norm of a feature too large for pieces, with weights that make something of it."""
    s = problem(82, count, F, H, n=500, m=400, norm=norm, sm=True, missing=True)
    if not norm:
        s["x_on"][:3, 2] = 1e5
        s["params"]["W1"][:, 2] *= 1e-5
    near(ctx, s, (0.1, 2, 3), count / 64)


@pytest.mark.parametrize("F", [8, 32, 48, 64, 100])
@pytest.mark.parametrize("norm, extra", [(True, True), (False, False)])
@pytest.mark.parametrize("H", [64, 128])
def test_several_tiles_of_predictions(ctx, H, norm, extra, F):
    s = problem(83, 70001, F, H, n=500, m=400, norm=norm, sm=extra, slow=extra, missing=True)
    exact, out = close.evaluate(s)[0], {k: torch.full((70001,), 7.0, device="cuda") for k in (("sigma", "sigma_slow") if extra else ("sigma",))}
    ctx.predict_pairs(predictor(ctx, s), *(dev(s[k]) for k in ("x_on", "x_off", "on", "off")), *out.values())
    for name, got in out.items():
        assert (abs(got.cpu().numpy() - exact[name]) <= 1e-5 * exact[name]).all(), name
