"""GPU: a predictor's loss with every gradient, and predictions of listed pairs, against the definition in float64; bounds come with
it (fit_reference)."""
import numpy as np
import pytest
import torch

import fit_reference as ref
import synth
from gpu_util import dev, dev_params, empty_matrix

pytestmark = pytest.mark.gpu

SM = (1, 2)
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    import paper_2303_13803_amd as mm
    c = mm.Context(64, 64)
    yield c
    c.close()


def problem(seed, count, F, H, n=50, m=40, norm=True, sm=False, slow=False, missing=False):
    """Features, a predictor, samples and targets (numpy)."""
    rng = np.random.default_rng(seed)
    params = synth.predictor_params(seed, F, H)
    if sm:
        params["W1sm"] = rng.normal(0, 0.2, H).astype(np.float32)
    if slow:
        params["W3slow"], params["b3slow"] = rng.normal(0, 0.2, H).astype(np.float32), rng.normal(0, 0.1, 1).astype(np.float32)
    if norm:
        params["ln_w"], params["ln_b"] = (1 + rng.normal(0, 0.2, 2 * F)).astype(np.float32), rng.normal(0, 0.2, 2 * F).astype(np.float32)
    s = {"params": params, "x_on": rng.random((n, F), dtype=np.float32), "x_off": rng.random((m, F), dtype=np.float32),
         "on": rng.integers(0, n, count).astype(np.int32), "off": rng.integers(0, m, count).astype(np.int32),
         "target": rng.random(count).astype(np.float32), "target_slow": rng.random(count).astype(np.float32) if slow else None,
         "sm": SM if sm else None, "eps": EPS if norm else None, "H": H}
    if missing:
        s["on"][rng.random(count) < 0.1] = -1
        s["off"][rng.random(count) < 0.1] = m
        s["target"][rng.random(count) < 0.2] = np.nan
        if slow:
            s["target_slow"][rng.random(count) < 0.2] = np.nan
    return s


def predictor(ctx, s):
    return ctx.predictor(dev_params(s["params"]), 1.0, sm=s["sm"], slow_limit=0.5 if s["target_slow"] is not None else None, norm_eps=s["eps"])


def call(ctx, s, drop=None, scale=None, want=True, pred=None):
    """What the library says: {name: numpy array}."""
    count = len(s["on"])
    pred = pred if pred is not None else predictor(ctx, s)
    slow = s["target_slow"] is not None
    out = {"loss": torch.full((1,), 7.0, device="cuda"), "sigma": torch.full((count,), 7.0, device="cuda")}
    if slow:
        out["sigma_slow"] = torch.full((count,), 7.0, device="cuda")
    grads = {k: torch.full(v.shape, 7.0, device="cuda") for k, v in s["params"].items()}
    work = torch.full((ctx.predictor_loss_work(pred, count),), 255, dtype=torch.uint8, device="cuda")       # NaN in every word
    ctx.predictor_loss(pred, dev(s["x_on"]), dev(s["x_off"]), dev(s["on"]), dev(s["off"]), dev(s["target"]), out["loss"], grads=grads if want else None,
                       target_slow=dev(s["target_slow"]) if slow else None, dropout=drop, scale=scale, sigma=out["sigma"], sigma_slow=out.get("sigma_slow"), work=work)
    if want:
        out.update(grads)
    return {k: v.cpu().numpy() for k, v in out.items()}


def definition(s, drop=None, scale=None):
    return ref.loss(s["params"], s["x_on"], s["x_off"], s["on"], s["off"], s["target"], 1.0 / max(len(s["on"]), 1) if scale is None else scale,
                    s["target_slow"], drop, s["sm"], s["eps"])


def compare(got, expected):
    for name, (value, bound) in expected.items():
        ref.within(got[name].reshape(value.shape), value, bound, name)
    assert set(expected) == set(got)


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("F", [3, 4, 16, 17, 31, 32, 33, 48, 64, 65, 128, 129, 200, 256])
def test_by_features(ctx, F, H):
    s = problem(F * H, 150, F, H, sm=F % 2 == 1, slow=F % 3 == 0)
    compare(call(ctx, s, (0.2, 5, 1)), definition(s, (0.2, 5, 1)))


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("count", [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 1000, 5003])
def test_by_samples(ctx, count, H):
    s = problem(count, count, 16, H, sm=True, slow=True)
    compare(call(ctx, s, (0.1, 1 << 60, 1 << 35)), definition(s, (0.1, 1 << 60, 1 << 35)))


@pytest.mark.parametrize("H", [64, 128])
def test_more_samples_than_the_device_holds_at_once(ctx, H):
    s = problem(9, 40007, 16, H, n=300, m=500)
    compare(call(ctx, s, (0.5, 3, 4)), definition(s, (0.5, 3, 4)))


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("sm", [False, True])
@pytest.mark.parametrize("slow", [False, True])
@pytest.mark.parametrize("drop", [None, (0.0, 1, 1), (0.3, 1, 1)])
def test_every_kind_of_predictor(ctx, norm, sm, slow, drop):
    """Also with samples that name no pair and targets nobody has measured."""
    s = problem(11, 333, 12, 64, norm=norm, sm=sm, slow=slow, missing=True)
    compare(call(ctx, s, drop), definition(s, drop if drop and drop[0] > 0 else None))


def test_one_workload_a_side_and_the_same_pair_again_and_again(ctx):
    s = problem(12, 700, 8, 128, n=1, m=1)
    compare(call(ctx, s, (0.1, 2, 3)), definition(s, (0.1, 2, 3)))


@pytest.mark.parametrize("which", ["nothing named", "nothing measured", "no workloads", "no samples"])
def test_nothing_to_learn_from(ctx, which):
    s = problem(13, 200, 8, 64, sm=True, slow=True)
    if which == "nothing named":
        s["on"][:] = -5
    if which == "nothing measured":
        s["target"][:] = s["target_slow"][:] = np.nan
    if which == "no workloads":
        s["x_on"] = s["x_on"][:0]
    if which == "no samples":
        for k in ("on", "off", "target", "target_slow"):
            s[k] = s[k][:0]
    got = call(ctx, s, (0.1, 2, 3))
    for name, value in got.items():
        if which != "nothing measured" or not name.startswith("sigma"):
            assert (value == 0).all(), name
        else:
            assert ((value > 0) & (value < 1)).all()


def test_indices_far_out_of_range(ctx):
    s = problem(14, 100, 8, 64)
    s["on"][::7], s["off"][::11] = np.iinfo(np.int32).max, np.iinfo(np.int32).min
    compare(call(ctx, s), definition(s))


def test_the_loss_alone_and_the_callers_scale(ctx):
    s = problem(15, 500, 16, 128, slow=True, missing=True)
    whole, alone = call(ctx, s, (0.1, 2, 3), 3.5), call(ctx, s, (0.1, 2, 3), 3.5, want=False)
    compare(whole, definition(s, (0.1, 2, 3), 3.5))
    # (the loss's partial sums are the same whether or not there are gradients)
    for name in alone:
        assert (alone[name] == whole[name]).all(), name


def test_the_same_call_gives_the_same_bits(ctx):
    s = problem(16, 30000, 32, 128, n=400, m=300, sm=True, slow=True)
    a, b = call(ctx, s, (0.1, 2, 3)), call(ctx, s, (0.1, 2, 3))
    for name in a:
        assert (a[name].view(np.int32) == b[name].view(np.int32)).all(), name


def test_units_that_never_fire_and_certain_predictions(ctx):
    """Every ReLU of the first layer closed; then predictions so sure that the logistic is 0 or 1 to the last bit."""
    s = problem(17, 200, 8, 64, norm=False)
    s["params"]["b1"][:] = -100.0
    compare(call(ctx, s), definition(s))
    s = problem(18, 200, 8, 64)
    s["params"]["W3"] *= 300.0
    got = call(ctx, s)
    assert all(np.isfinite(v).all() for v in got.values())
    s["params"]["b3"][:] = 200.0
    s["params"]["W3"][:] = 0.0
    got = call(ctx, s)
    assert (got["sigma"] == 1.0).all() and (got["W2"] == 0).all() and (got["b3"] == 0).all()


def test_features_of_a_thousand_scales(ctx):
    """A feature in microseconds beside fractions: what a norm is there for; and rows that are all the same value."""
    s = problem(19, 300, 16, 64)
    s["x_on"][:, 3] *= 1000.0
    s["x_off"][:5] = 0.25
    compare(call(ctx, s), definition(s))


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("F", [1, 2, 7, 49, 63, 255])
def test_by_odd_features_without_an_sm_share(ctx, F, H):
    s = problem(F + H, 97, F, H, norm=F % 3 > 0, missing=True)
    compare(call(ctx, s, (0.25, 9, 9)), definition(s, (0.25, 9, 9)))


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("F", [5, 40])
@pytest.mark.parametrize("largest", [100.0, 4096.0, 4097.0, 1e7, 1e12])
@pytest.mark.parametrize("drop", [None, (0.2, 3, 3)])
def test_a_few_large_features_without_a_norm(ctx, F, H, largest, drop):
    """Beside features of about 1, which keep their precision; with weights that make something of both."""
    s = problem(30, 210, F, H, norm=False)
    s["x_on"][:3, 2] = largest
    s["params"]["W1"][:, 2] /= np.float32(largest)
    compare(call(ctx, s, drop), definition(s, drop))
    sigma = torch.full((210,), 7.0, device="cuda")
    ctx.predict_pairs(predictor(ctx, s), dev(s["x_on"]), dev(s["x_off"]), dev(s["on"]), dev(s["off"]), sigma)
    ref.within(sigma.cpu().numpy(), *definition(s)["sigma"], "sigma")


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("largest", [100.0, 1e7])
def test_a_large_sm_share(ctx, largest, norm):
    s = problem(31, 210, 8, 64, norm=norm, sm=True, slow=True)
    s["x_on"][:3, SM[0]], s["x_off"][:3, SM[1]] = -largest, largest
    s["params"]["W1sm"] /= np.float32(largest)
    compare(call(ctx, s, (0.2, 3, 3)), definition(s, (0.2, 3, 3)))


@pytest.mark.parametrize("norm", [False, True])
def test_many_predictions_of_the_same_pairs(ctx, norm):
    """More than a workgroup looks up by itself; every pair of 50 and 40 workloads again and again."""
    s = problem(38, 2000, 8, 128, norm=norm, sm=True)
    s["on"], s["off"] = np.repeat(np.arange(50), 40).astype(np.int32), np.tile(np.arange(40), 50).astype(np.int32)
    which = np.random.default_rng(38).integers(0, 2000, 700001)
    sigma = torch.full((700001,), 7.0, device="cuda")
    ctx.predict_pairs(predictor(ctx, s), dev(s["x_on"]), dev(s["x_off"]), dev(s["on"][which]), dev(s["off"][which]), sigma)
    value, bound = definition(s)["sigma"]
    ref.within(sigma.cpu().numpy(), value[which], bound[which], "sigma")


def test_large_features_that_no_sample_names(ctx):
    """Whether they are looked at or not (few samples, many samples): predictions of the others do not change beyond their bounds."""
    for count in (20, 2000):
        s = problem(32, count, 16, 128, norm=False)
        s["x_on"][7], s["x_off"][9] = 1e20, np.inf
        s["on"][s["on"] == 7], s["off"][s["off"] == 9] = 8, 8
        compare(call(ctx, s), definition(s))


@pytest.mark.parametrize("H", [64, 128])
def test_targets_far_from_what_a_logistic_gives(ctx, H):
    s = problem(33, 500, 16, H, slow=True)
    s["target"] = (s["target"] * 60 - 10).astype(np.float32)
    s["target_slow"][::50] = -40.0
    compare(call(ctx, s, (0.1, 4, 4)), definition(s, (0.1, 4, 4)))


@pytest.mark.parametrize("p", [2.0 ** -16, 0.99, 65535 / 65536])
def test_hardly_any_dropout_and_hardly_anything_left(ctx, p):
    s = problem(34, 400, 16, 128)
    compare(call(ctx, s, (p, 4, 4)), definition(s, (p, 4, 4)))


def test_weights_that_are_all_zero(ctx):
    s = problem(35, 100, 16, 64)
    for k in s["params"]:
        s["params"][k][:] = 0.0
    compare(call(ctx, s), definition(s))


@pytest.mark.parametrize("F", [16, 100])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_a_feature_that_is_not_finite_shows_where_it_is_used(ctx, F, norm, value):
    s = problem(36, 300, F, 64, norm=norm)
    s["x_off"][5, 3] = value
    s["off"][:10] = 5
    got = call(ctx, s)
    used = s["off"] == 5
    assert np.isnan(got["loss"]).all() and np.isfinite(got["sigma"][~used]).all()
    if norm or np.isnan(value):
        assert np.isnan(got["sigma"][used]).all()
    else:                                                   # (without a norm it may also make the logistic certain)
        assert (np.isnan(got["sigma"][used]) | (got["sigma"][used] == 0) | (got["sigma"][used] == 1)).all()


def test_predictions_without_workloads(ctx):
    s = problem(37, 70, 8, 64, slow=True)
    pred = predictor(ctx, s)
    none = torch.empty((0, 8), device="cuda")
    for x_on, x_off in ((none, dev(s["x_off"])), (dev(s["x_on"]), none), (none, none)):
        sigma, slow = (torch.full((70,), 7.0, device="cuda") for _ in range(2))
        ctx.predict_pairs(pred, x_on, x_off, dev(s["on"]), dev(s["off"]), sigma, slow)
        assert (sigma == 0).all() and (slow == 0).all()


def test_a_fit_that_has_diverged_shows(ctx):
    s = problem(20, 100, 8, 64)
    s["params"]["W1"][3, 2] = np.nan
    got = call(ctx, s)
    assert np.isnan(got["loss"]).all() and np.isnan(got["sigma"]).all()


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("norm, sm, slow", [(True, True, True), (False, False, False), (True, False, False)])
def test_losses_differ_as_the_gradient_says(ctx, H, norm, sm, slow):
    """Along its own direction the loss changes by what the gradient says; the quotient's own error is taken from the
    definition at the same places, and what is left is what both losses may be off."""
    s = problem(21, 800, 16, H, norm=norm, sm=sm, slow=slow)
    drop = (0.2, 7, 7)
    g = {k: v for k, v in call(ctx, s, drop).items() if k in s["params"]}
    square = sum(float((v.astype(np.float64) ** 2).sum()) for v in g.values())
    assert square > 0
    step, losses, exact = 0.01 / np.sqrt(square), [], []
    for sign in (1, -1):
        moved = dict(s, params={k: (v + sign * step * g[k].reshape(v.shape)).astype(np.float32) for k, v in s["params"].items()})
        losses.append(float(call(ctx, moved, drop, want=False)["loss"][0]))
        exact.append(definition(moved, drop)["loss"])
    slope = (losses[0] - losses[1]) / (2 * step)
    room = (exact[0][1][0] + exact[1][1][0] + 4 * ref.U * exact[0][0][0]) / (2 * step)
    assert abs(slope - (exact[0][0][0] - exact[1][0][0]) / (2 * step)) <= room
    # a central difference over a hundredth of a unit's length: curvature changes the slope by a few parts in a hundred
    assert abs(slope - square) < 0.05 * square


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("count, F", [(1, 16), (5, 3), (64, 32), (1000, 33), (777, 256)])
def test_predictions_of_listed_pairs(ctx, count, F, H):
    s = problem(count + F, count, F, H, sm=True, slow=True, missing=count > 5)
    pred = predictor(ctx, s)
    sigma, slow = (torch.full((count,), 7.0, device="cuda") for _ in range(2))
    ctx.predict_pairs(pred, dev(s["x_on"]), dev(s["x_off"]), dev(s["on"]), dev(s["off"]), sigma, slow)
    expected = definition(s)
    for got, name in ((sigma, "sigma"), (slow, "sigma_slow")):
        ref.within(got.cpu().numpy(), *expected[name], name)
    only = torch.full((count,), 7.0, device="cuda")
    ctx.predict_pairs(pred, dev(s["x_on"]), dev(s["x_off"]), dev(s["on"]), dev(s["off"]), only)
    assert torch.equal(only, sigma)


@pytest.mark.parametrize("count, H", [(1024, 128), (1025, 128), (2048, 64), (2049, 64)])
def test_predictions_about_as_many_as_the_device_holds(ctx, count, H):
    s = problem(count, count, 12, H, n=300, m=200, sm=True, slow=True, missing=True)
    sigma, slow = (torch.full((count,), 7.0, device="cuda") for _ in range(2))
    ctx.predict_pairs(predictor(ctx, s), dev(s["x_on"]), dev(s["x_off"]), dev(s["on"]), dev(s["off"]), sigma, slow)
    expected = definition(s)
    for got, name in ((sigma, "sigma"), (slow, "sigma_slow")):
        ref.within(got.cpu().numpy(), *expected[name], name)


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("F", [1, 2, 5, 6, 63, 64, 65, 130, 255])
def test_single_predictions_by_features(ctx, F, norm, H):
    """A few pairs, an infinity and a NaN among their features."""
    s = problem(40 + F, 9, F, H, norm=norm)
    s["x_on"][49], s["x_off"][39, F - 1] = np.nan, np.inf
    s["on"][:7], s["off"][:7] = [0, 1, 49, 3, -1, 5, 50], [0, 1, 2, 39, 4, 40, 6]
    s["on"][7:], s["off"][7:] = 8, 9
    sigma = torch.full((9,), 7.0, device="cuda")
    ctx.predict_pairs(predictor(ctx, s), dev(s["x_on"]), dev(s["x_off"]), dev(s["on"]), dev(s["off"]), sigma)
    got, good = sigma.cpu().numpy(), [0, 1, 4, 5, 6, 7, 8]
    with np.errstate(invalid="ignore"):
        value, bound = definition(s)["sigma"]
    ref.within(got[good], value[good], bound[good], "sigma")
    assert np.isnan(got[2]) and (np.isnan(got[3]) or not norm and got[3] in (0.0, 1.0)) and (got[4:7] == 0).all()


@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("split", [0, 1])
def test_scores_of_a_predictor_with_a_norm(ctx, H, split):
    """Every pair through mf_score_pairs: within 1e-5 of the definition (as without a norm), the mask from the features as they are."""
    import paper_2303_13803_amd as mm
    n, m, F = 61, 64, 19
    s = problem(22, n * m, F, H, n=n, m=m, sm=True)
    s["on"], s["off"] = np.repeat(np.arange(n), m).astype(np.int32), np.tile(np.arange(m), n).astype(np.int32)
    W, sigma = empty_matrix(n, m), torch.empty((n, m), device="cuda")
    ctx.set_option("score_split", split)
    pred = ctx.predictor(dev_params(s["params"]), 2.0 ** 20, sm=SM, norm_eps=EPS)
    ctx.score_pairs(pred, dev(s["x_on"]), dev(s["x_off"]), W, sigma)
    value = definition(s)["sigma"][0].reshape(n, m)
    assert (np.abs(sigma.cpu().numpy() - value) <= 1e-5 * value).all()
    mask = s["x_on"][:, None, 0] + s["x_off"][None, :, 0] > np.float32(1.0)
    W1 = W[:, :m].cpu().numpy()
    assert ((W1 == mm.INFEASIBLE) == mask).all()
    W2 = empty_matrix(n, m)
    ctx.score_pairs(pred, dev(s["x_on"]), dev(s["x_off"]), W2)              # in memory order
    assert torch.equal(W2[:, :m], W[:, :m])
    listed = torch.empty(n * m, device="cuda")
    ctx.predict_pairs(pred, dev(s["x_on"]), dev(s["x_off"]), dev(s["on"]), dev(s["off"]), listed)
    assert (np.abs(listed.cpu().numpy().reshape(n, m) - value) <= 1e-5 * value).all()
    ctx.set_option("score_split", 1)


def test_typed_scores_with_and_without_a_norm(ctx):
    """One GPU type's predictor has a norm and the other's has not."""
    n, m, F = 40, 33, 8
    a, b = problem(23, 1, F, 64, n=n, m=m), problem(24, 1, F, 128, n=n, m=m, norm=False)
    preds = [ctx.predictor(dev_params(a["params"]), 2.0 ** 20, norm_eps=EPS), ctx.predictor(dev_params(b["params"]), 2.0 ** 20)]
    types = (np.arange(n) % 2).astype(np.int32)
    W, sigma = empty_matrix(n, m), torch.empty((n, m), device="cuda")
    ctx.score_pairs_typed(preds, dev(types), dev(a["x_on"]), dev(a["x_off"]), W, sigma)
    for t, s in ((0, a), (1, b)):
        rows = np.flatnonzero(types == t)
        s = dict(s, x_on=a["x_on"], x_off=a["x_off"], on=np.repeat(rows, m).astype(np.int32), off=np.tile(np.arange(m), len(rows)).astype(np.int32), target=None)
        value = definition(s)["sigma"][0].reshape(len(rows), m)
        assert (np.abs(sigma.cpu().numpy()[rows] - value) <= 1e-5 * value).all()


def test_a_fit_then_a_round(ctx, orc):
    """All of it as it is used: steps of momentum descent captured once and replayed, the step counted on the device; every replay's
    loss and gradients are those of an eager call; then a round is scheduled with what was learnt, from rows whose memory order the
    mask takes from the features as they are."""
    import paper_2303_13803_amd as mm
    n, m, F, H, count = 48, 64, 16, 64, 600
    s = problem(25, count, F, H, n=n, m=m, missing=True)
    params = dev_params(s["params"])
    x_on, x_off, on, off, target = (dev(s[k]) for k in ("x_on", "x_off", "on", "off", "target"))
    stream = torch.cuda.Stream()
    mine = mm.Context(1, 1, stream=stream)
    pred, grads = mine.predictor(params, 2.0 ** 20, norm_eps=EPS), {k: torch.empty_like(v) for k, v in params.items()}
    loss, step, speed = torch.empty(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), {k: torch.zeros_like(v) for k, v in params.items()}
    work = torch.empty(mine.predictor_loss_work(pred, count), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        mine.predictor_loss(pred, x_on, x_off, on, off, target, loss, grads=grads, dropout=(0.1, 99, step), work=work)
    eager, again = torch.empty(1, device="cuda"), {k: torch.empty_like(v) for k, v in params.items()}
    losses = []
    for k in range(30):
        graph.replay()
        torch.cuda.synchronize()
        ctx.predictor_loss(ctx.predictor(params, 2.0 ** 20, norm_eps=EPS), x_on, x_off, on, off, target, eager, grads=again, dropout=(0.1, 99, k))
        torch.cuda.synchronize()
        assert torch.equal(loss, eager) and all(torch.equal(grads[q], again[q]) for q in grads), k
        for q in params:
            speed[q].mul_(0.9).add_(grads[q])
            params[q].add_(speed[q], alpha=-0.05)
        step.add_(1)
        losses.append(float(loss[0]))
        torch.cuda.synchronize()
    assert all(np.isfinite(losses))
    W, r2c = empty_matrix(n, m), torch.empty(n, dtype=torch.int32, device="cuda")
    u, v = torch.empty(n, dtype=torch.int64, device="cuda"), torch.empty(m, dtype=torch.int64, device="cuda")
    res = ctx.schedule_round(ctx.predictor(params, 2.0 ** 20, norm_eps=EPS), x_on, x_off, W, r2c, u, v)
    Wh = W[:, :m].cpu().numpy()
    learnt = dict(s, params={k: p.cpu().numpy() for k, p in params.items()}, on=np.repeat(np.arange(n), m).astype(np.int32),
                  off=np.tile(np.arange(m), n).astype(np.int32), target=None)
    value = definition(learnt)["sigma"][0].reshape(n, m)
    fits = s["x_on"][:, None, 0] + s["x_off"][None, :, 0] <= np.float32(1.0)
    assert ((Wh != mm.INFEASIBLE) == fits).all()
    assert (np.abs(Wh[fits] - 2.0 ** 20 * value[fits]) <= 1e-5 * 2.0 ** 20 + 1).all()
    assert res.primal == orc.max_weight_matching(Wh)[0] and res.cert_ok == 1
    mine.close()


def test_an_update_scores_again_with_the_norm(ctx):
    """mf_schedule_round_update's rows and columns are those of a whole pass."""
    n, m, F = 50, 60, 8
    s = problem(26, 1, F, 64, n=n, m=m)
    pred = ctx.predictor(dev_params(s["params"]), 2.0 ** 20, norm_eps=EPS)
    W = empty_matrix(n, m)
    r2c, u, v = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int64, device="cuda"), torch.empty(m, dtype=torch.int64, device="cuda")
    ctx.schedule_round(pred, dev(s["x_on"]), dev(s["x_off"]), W, r2c, u, v)
    rng = np.random.default_rng(1)
    rows, cols = np.array([3, 40], dtype=np.int32), np.array([0, 59, 7], dtype=np.int32)
    s["x_on"][rows], s["x_off"][cols] = rng.random((2, F), dtype=np.float32), rng.random((3, F), dtype=np.float32)
    ctx.schedule_round_update(pred, dev(s["x_on"]), dev(s["x_off"]), dev(rows), dev(cols), W, r2c, u, v)
    fresh = empty_matrix(n, m)
    ctx.schedule_round(pred, dev(s["x_on"]), dev(s["x_off"]), fresh, r2c, u, v)
    assert torch.equal(W[:, :m], fresh[:, :m])


def shifted(t):
    """The same values, beginning four bytes beyond a multiple of sixteen."""
    buf = torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")
    out = buf[1:1 + t.numel()].view(t.shape)
    assert out.data_ptr() % 16 == 4
    return out.copy_(t)


@pytest.mark.parametrize("H, F, norm, count", [(64, 16, True, 300), (128, 32, True, 300), (64, 50, False, 300), (128, 70, True, 300), (64, 16, True, 5000), (128, 17, False, 5000)])
def test_tensors_that_begin_anywhere(ctx, H, F, norm, count):
    """Features, samples, weights but those of the hidden layer and the output unit, and gradients, aligned to nothing but their values."""
    s = problem(50, count, F, H, norm=norm, slow=True)
    params = {k: v if k in ("W2", "b2", "W3", "W3slow") else shifted(v) for k, v in dev_params(s["params"]).items()}
    pred = ctx.predictor(params, 1.0, slow_limit=0.5, norm_eps=s["eps"])
    x_on, x_off, on, off, target, slow = (shifted(dev(s[k])) for k in ("x_on", "x_off", "on", "off", "target", "target_slow"))
    out = {"loss": shifted(torch.zeros(1, device="cuda")), "sigma": shifted(torch.zeros(count, device="cuda")), "sigma_slow": shifted(torch.zeros(count, device="cuda"))}
    grads = {k: shifted(torch.zeros(v.shape, device="cuda")) for k, v in s["params"].items()}
    ctx.predictor_loss(pred, x_on, x_off, on, off, target, out["loss"], grads=grads, target_slow=slow, sigma=out["sigma"], sigma_slow=out["sigma_slow"])
    compare({k: v.cpu().numpy() for k, v in {**out, **grads}.items()}, definition(s))
    sigma = shifted(torch.zeros(count, device="cuda"))
    ctx.predict_pairs(pred, x_on, x_off, on, off, sigma)
    ref.within(sigma.cpu().numpy(), *definition(s)["sigma"], "sigma")


def test_two_graphs_of_a_context_replayed_in_turn(ctx):
    """Both use the context's scratch: one predictor has many features, the other no norm; with eager calls of the context between them."""
    import paper_2303_13803_amd as mm
    stream = torch.cuda.Stream()
    mine = mm.Context(1, 1, stream=stream)
    problems = [problem(60, 700, 100, 64, missing=True), problem(61, 900, 20, 64, norm=False, sm=True), problem(62, 800, 30, 64, sm=True)]
    calls, expected, graphs = [], [call(ctx, s, (0.1, 2, 3)) for s in problems], []
    for s in problems:
        pred, t = predictor(mine, s), {k: dev(s[k]) for k in ("x_on", "x_off", "on", "off", "target")}
        out = {"loss": torch.zeros(1, device="cuda"), "grads": {k: torch.zeros(v.shape, device="cuda") for k, v in s["params"].items()},
               "sigma": torch.zeros(len(s["on"]), device="cuda"), "work": torch.empty(mine.predictor_loss_work(pred, len(s["on"])), dtype=torch.uint8, device="cuda")}
        calls.append((pred, t, out))
    torch.cuda.synchronize()
    for pred, t, out in calls[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            mine.predictor_loss(pred, **t, **out, dropout=(0.1, 2, 3))
    for _ in range(3):
        for pred, t, out in calls:
            out["loss"].zero_()
            out["sigma"].zero_()
            for g in out["grads"].values():
                g.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graphs[0].replay()
            mine.predictor_loss(calls[2][0], **calls[2][1], **calls[2][2], dropout=(0.1, 2, 3))
            graphs[1].replay()
        torch.cuda.synchronize()
        for (_, _, out), e in zip(calls, expected):
            assert (out["loss"].cpu().numpy() == e["loss"]).all() and (out["sigma"].cpu().numpy() == e["sigma"]).all()
            for k, g in out["grads"].items():
                assert (g.cpu().numpy() == e[k]).all(), k
    mine.close()


def test_scratch_of_the_librarys_own_in_the_order_of_its_stream(ctx):
    """A context on a stream that is not the current one, and no scratch given: what the allocator hands out next on the current stream is another's."""
    import paper_2303_13803_amd as mm
    mine = mm.Context(1, 1, stream=torch.cuda.Stream())
    s = problem(63, 20000, 32, 128, n=300, m=300)
    expected = call(ctx, s, (0.1, 2, 3))
    t, pred = {k: dev(s[k]) for k in ("x_on", "x_off", "on", "off", "target")}, predictor(mine, s)
    loss, grads = torch.zeros(1, device="cuda"), {k: torch.zeros(v.shape, device="cuda") for k, v in s["params"].items()}
    torch.cuda.synchronize()
    for _ in range(3):
        mine.predictor_loss(pred, **t, loss=loss, grads=grads, dropout=(0.1, 2, 3))
        torch.full((mine.predictor_loss_work(pred, 20000),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert (loss.cpu().numpy() == expected["loss"]).all() and all((g.cpu().numpy() == expected[k]).all() for k, g in grads.items())
    mine.close()


def test_two_contexts_at_once(ctx):
    """Two fits on two streams, each with its own scratch."""
    import paper_2303_13803_amd as mm
    s, t = problem(27, 20000, 32, 128, n=300, m=300), problem(28, 20000, 16, 64, n=300, m=300)
    expected = [call(ctx, s, (0.1, 2, 3)), call(ctx, t, (0.1, 2, 3))]
    contexts = [mm.Context(1, 1, stream=torch.cuda.Stream()) for _ in range(2)]
    inputs = [{k: dev(q[k]) for k in ("x_on", "x_off", "on", "off", "target")} for q in (s, t)]
    preds = [predictor(c, q) for c, q in zip(contexts, (s, t))]
    losses = [torch.empty(1, device="cuda") for _ in range(2)]
    grads = [{k: torch.empty(v.shape, device="cuda") for k, v in q["params"].items()} for q in (s, t)]
    works = [torch.empty(c.predictor_loss_work(p, 20000), dtype=torch.uint8, device="cuda") for c, p in zip(contexts, preds)]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, p, i, l, g, w in zip(contexts, preds, inputs, losses, grads, works):
            c.predictor_loss(p, **i, loss=l, grads=g, dropout=(0.1, 2, 3), work=w)
    torch.cuda.synchronize()
    for e, l, g in zip(expected, losses, grads):
        assert (e["loss"] == l.cpu().numpy()).all()
        for k in g:
            assert (e[k] == g[k].cpu().numpy()).all(), k
    for c in contexts:
        c.close()


def test_a_fit_refuses_tensors_that_do_not_fit(ctx):
    s = problem(29, 64, 8, 64, slow=True)
    pred = predictor(ctx, s)
    x_on, x_off, on, off, target, slow = (dev(s[k]) for k in ("x_on", "x_off", "on", "off", "target", "target_slow"))
    loss, grads = torch.empty(1, device="cuda"), {k: torch.empty(v.shape, device="cuda") for k, v in s["params"].items()}
    good = dict(pred=pred, x_on=x_on, x_off=x_off, on=on, off=off, target=target, loss=loss, grads=grads, target_slow=slow)
    ctx.predictor_loss(**good)
    for change in ({"on": on.long()}, {"on": on[:5]}, {"off": off.cpu()}, {"x_on": x_on[:, :5]}, {"x_on": x_on.double()}, {"x_off": x_off.t()}, {"target": target[::2]},
                   {"target": None}, {"loss": grads["W3"]}, {"grads": dict(grads, W2=grads["W1"])}, {"sigma": target[:3]}, {"work": target}):
        with pytest.raises((TypeError, ValueError)):
            ctx.predictor_loss(**dict(good, **change))
    with pytest.raises(KeyError):
        ctx.predictor_loss(**dict(good, grads={k: v for k, v in grads.items() if k != "W3slow"}))
    from paper_2303_13803_amd import MuxmatchError
    for change in ({"target_slow": None}, {"scale": 0.0}, {"dropout": (1.0, 5)}, {"work": torch.empty(64, dtype=torch.uint8, device="cuda")}):
        with pytest.raises(MuxmatchError):
            ctx.predictor_loss(**dict(good, **change))
    with pytest.raises(ValueError):
        ctx.predict_pairs(pred, x_on, x_off, on, off, loss)
