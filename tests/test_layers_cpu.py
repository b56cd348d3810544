"""Layers and the predictor's loss without a device: random bits against published answers, the oracle's gradients against
differences, and what the calls refuse."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

import fit_reference as ref
import synth

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2303_13803_amd", "csrc")


@pytest.mark.skipif(not shutil.which("g++"), reason="no g++")
def test_random_bits_and_limits(tmp_path):
    """The header's blocks are the answers published with the generator, and its limits are those of rint."""
    done = subprocess.run(["g++", "-O1", "-Wall", "-Wno-unknown-pragmas", "-I", CSRC, "-o", str(tmp_path / "philox"), os.path.join(ROOT, "tests", "philox.cpp")],
                          capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    done = subprocess.run([str(tmp_path / "philox")], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


def test_the_oracle_has_the_published_bits():
    """Key and counter zero: 6627e8d5 e169c58d bc57ac4c 9b00dbd8."""
    bits = ref.random_bits(0, 0, 0, 8)
    words = [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert bits.tolist() == [h for w in words for h in (w & 0xFFFF, w >> 16)]


def test_about_the_asked_share_is_dropped():
    """Of a million elements: a binomial deviation is 0.0005 at most, and five of them are not seen by chance."""
    for p in (0.1, 0.5, 0.9):
        k = ref.kept(1000, 1000, p, 77, 5, 1)
        assert abs((k == 0).mean() - p) < 5 * 0.0005 and abs(k.mean() - 1) < 5 * 0.0005 / (1 - p)


def _problem(seed, count=37, F=5, H=64, sm=True, slow=True, norm=True):
    rng = np.random.default_rng(seed)
    params = synth.predictor_params(seed, F, H)
    if sm:
        params["W1sm"] = rng.normal(0, 0.2, H).astype(np.float32)
    if slow:
        params["W3slow"], params["b3slow"] = rng.normal(0, 0.2, H).astype(np.float32), rng.normal(0, 0.1, 1).astype(np.float32)
    if norm:
        params["ln_w"], params["ln_b"] = (1 + rng.normal(0, 0.2, 2 * F)).astype(np.float32), rng.normal(0, 0.2, 2 * F).astype(np.float32)
    x_on, x_off = rng.random((11, F), dtype=np.float32), rng.random((7, F), dtype=np.float32)
    on, off = rng.integers(-1, 12, count).astype(np.int32), rng.integers(0, 7, count).astype(np.int32)
    target, slowdown = rng.random(count), rng.random(count)
    target[::5] = slowdown[::3] = np.nan
    return params, x_on, x_off, on, off, target, slowdown


@pytest.mark.parametrize("norm, sm, slow, drop", [(True, True, True, (0.3, 9, 2)), (False, False, False, None), (True, False, True, None)])
def test_the_oracles_gradients_are_those_of_differences(norm, sm, slow, drop):
    """In float64 a central difference with a step of 1e-5 is good to about 1e-9; a ReLU that changes sides in between costs more, at few places."""
    params, x_on, x_off, on, off, target, slowdown = _problem(3, norm=norm, sm=sm, slow=slow)
    rng = np.random.default_rng(4)
    at = lambda q: ref.loss(q, x_on, x_off, on, off, target, 1 / 37, slowdown if slow else None, drop, (1, 2) if sm else None, 1e-5 if norm else None)
    g = at(params)
    for name, value in params.items():
        for _ in range(4):
            k = rng.integers(value.size)
            moved = []
            for h in (1e-5, -1e-5):
                q = {n: np.asarray(v, dtype=np.float64).copy() for n, v in params.items()}
                q[name].reshape(-1)[k] += h
                moved.append(at(q)["loss"][0][0])
            slope = (moved[0] - moved[1]) / 2e-5
            assert abs(slope - g[name][0].reshape(-1)[k]) < 1e-7, (name, k)


@pytest.mark.parametrize("eps", [1e-5, 1e-2])
def test_the_oracles_norm_gradients_are_those_of_differences(eps):
    rng = np.random.default_rng(5)
    x, dy, w, b = rng.normal(size=(3, 7)), rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=7)
    at = lambda x, w, b: (ref.norm_rows(x, w, b, eps)[0] * dy).sum()
    dx, _, dw, _, db, _ = ref.norm_grad_rows(x, dy, w, eps)
    for got, which in ((dx, 0), (dw, 1), (db, 2)):
        for k in range(got.size):
            moved = []
            for h in (1e-6, -1e-6):
                args = [x.copy(), w.copy(), b.copy()]
                args[which].reshape(-1)[k] += h
                moved.append(at(*args))
            assert abs((moved[0] - moved[1]) / 2e-6 - got.reshape(-1)[k]) < 1e-7


# ---- what is refused.  A refused call touches neither the device nor anything its pointers name, so a context that was never
# created (zeros) and made-up addresses do.

@pytest.fixture(scope="module")
def lib():
    from paper_2303_13803_amd import binding
    return binding


@pytest.fixture(scope="module")
def ctx():
    return C.cast(C.create_string_buffer(1 << 16), C.c_void_p)


A = 0x10000         # an address like any other, 16-byte aligned


def _norm(**change):
    a = dict(type=0, x=A, rows=3, width=8, ldx=8, w=A, b=A, eps=1e-5, y=A, ldy=8)
    return list({**a, **change}.values())


@pytest.mark.parametrize("change", [
    {"type": 3}, {"type": -1}, {"x": None}, {"rows": -1}, {"width": 0}, {"ldx": 7}, {"w": None}, {"b": None}, {"eps": 0.0}, {"eps": -1.0}, {"eps": float("nan")},
    {"eps": float("inf")}, {"y": None}, {"ldy": 7}, {"x": A + 2}, {"y": A + 1}, {"w": A + 2}, {"type": 1, "x": A + 1}, {"ldx": 1 << 62}])
def test_layer_norm_refuses(lib, ctx, change):
    assert lib.raw_library().mf_layer_norm(ctx, *_norm(**change)) == lib.ERR_ARG


def test_sizes_beyond_what_the_layers_support(lib, ctx):
    raw = lib.raw_library()
    assert raw.mf_layer_norm(ctx, *_norm(width=8193, ldx=8193, ldy=8193)) == lib.ERR_SHAPE
    assert raw.mf_layer_norm(ctx, *_norm(rows=1 << 46)) == lib.ERR_SHAPE
    assert raw.mf_layer_norm_grad_work(ctx, 10, 8193) == lib.ERR_SHAPE and raw.mf_layer_norm_grad_work(ctx, -1, 8) == lib.ERR_ARG
    assert raw.mf_layer_norm_grad_work(None, 10, 8) == lib.ERR_ARG and raw.mf_layer_norm(None, *_norm()) == lib.ERR_ARG
    assert raw.mf_layer_norm(ctx, *_norm(rows=0, x=None, y=None)) == lib.OK           # nothing to do


@pytest.mark.parametrize("change", [{"dy": None}, {"lddy": 7}, {"dx": None}, {"lddx": 5}, {"dw": None}, {"db": None}, {"work": None}, {"work": A + 8}, {"bytes": 2 * 8 * 4 - 1},
                                    {"eps": 0.0}, {"dw": A + 2}, {"dx": A + 2}])
def test_layer_norm_grad_refuses(lib, ctx, change):
    a = dict(type=0, x=A, rows=3, width=8, ldx=8, dy=A, lddy=8, w=A, eps=1e-5, dx=A, lddx=8, dw=A, db=A, work=A, bytes=1 << 20)
    assert lib.raw_library().mf_layer_norm_grad_work(ctx, 3, 8) == 2 * 8 * 4
    assert lib.raw_library().mf_layer_norm_grad(ctx, *{**a, **change}.values()) == lib.ERR_ARG


@pytest.mark.parametrize("change, rule", [
    ({}, {"p": 1.0}), ({}, {"p": -0.1}), ({}, {"p": float("nan")}), ({}, {"p": 1 - 2 ** -18}), ({"layer": -1}, {}), ({"layer": 65536}, {}), ({"x": None}, {}),
    ({"y": None}, {}), ({"ldx": 7}, {}), ({"type": 5}, {}), ({"rule": None}, {}), ({}, {"d_step": A + 4})])
def test_dropout_refuses(lib, ctx, change, rule):
    r = lib.DropoutRule(*{**dict(p=0.5, seed=1, step=2, d_step=None), **rule}.values())
    a = dict(type=0, x=A, rows=3, width=8, ldx=8, rule=C.byref(r), layer=0, y=A, ldy=8)
    assert lib.raw_library().mf_dropout(ctx, *{**a, **change}.values()) == lib.ERR_ARG


def test_layers_refuse_to_write_in_place_with_another_pitch(lib, ctx):
    raw, rule = lib.raw_library(), lib.DropoutRule(0.5, 1, 2, None)
    assert raw.mf_layer_norm(ctx, *_norm(ldy=9)) == lib.ERR_ARG
    assert raw.mf_dropout(ctx, 0, A, 3, 8, 9, C.byref(rule), 0, A, 8) == lib.ERR_ARG
    for x, ldx, dy, lddy, dx, lddx in ((A, 8, 2 * A, 8, A, 9), (A, 8, 2 * A, 9, 2 * A, 8)):
        assert raw.mf_layer_norm_grad(ctx, 0, x, 3, 8, ldx, dy, lddy, A, 1e-5, dx, lddx, A, A, A, 1 << 20) == lib.ERR_ARG


def _predictor(lib, **change):
    p = dict(F=16, H=64, scale=1.0, mem_feature=0, mem_limit=1.0, d_W1=A, d_b1=A, d_W2=A, d_b2=A, d_W3=A, d_b3=A, d_W1sm=None, sm_on_feature=0, sm_off_feature=0,
             d_W3_slow=None, d_b3_slow=None, slow_limit=0.0, d_ln_w=A, d_ln_b=A, ln_eps=1e-5)
    return lib.Predictor(*{**p, **change}.values())


def _loss(lib, ctx, pred=(), samples=(), grads=(), **change):
    p = _predictor(lib, **dict(pred))
    s = lib.Samples(*{**dict(d_on=A, d_off=A, d_target=A, d_target_slow=None, count=100), **dict(samples)}.values())
    g = lib.Gradients(*{**{m: A for m, *_ in lib.PARAMETERS}, **dict(grads)}.values())
    a = dict(predictor=C.byref(p), x_on=A, n=5, x_off=A, m=5, listed=C.byref(s), dropout=None, scale=0.01, grads=C.byref(g), loss=A, sigma=A, sigma_slow=None,
             work=A, bytes=1 << 30)
    return lib.raw_library().mf_predictor_loss(ctx, *{**a, **change}.values())


@pytest.mark.parametrize("pred, samples, grads, change", [
    ({"d_ln_b": None}, {}, {}, {}), ({"ln_eps": 0.0}, {}, {}, {}), ({"ln_eps": float("nan")}, {}, {}, {}), ({"H": 96}, {}, {}, {}), ({"F": 0}, {}, {}, {}), ({"F": 257}, {}, {}, {}),
    ({"d_W2": A + 4}, {}, {}, {}), ({"d_W1sm": A, "sm_on_feature": 16}, {}, {}, {}), ({"d_W3_slow": A, "d_b3_slow": A}, {}, {}, {}),
    ({}, {"d_on": None}, {}, {}), ({}, {"d_off": None}, {}, {}), ({}, {"d_target": None}, {}, {}), ({}, {"d_target_slow": A}, {}, {}), ({}, {"count": -1}, {}, {}),
    ({}, {"d_on": A + 1}, {}, {}), ({}, {}, {"d_W1": None}, {}), ({}, {}, {"d_b3": None}, {}), ({}, {}, {"d_ln_w": None}, {}), ({}, {}, {"d_ln_b": A + 2}, {}),
    ({"d_W1sm": A}, {}, {"d_W1sm": None}, {}),
    ({}, {}, {}, {"x_on": None}), ({}, {}, {}, {"n": -1}), ({}, {}, {}, {"m": -3}), ({}, {}, {}, {"scale": 0.0}), ({}, {}, {}, {"scale": float("inf")}), ({}, {}, {}, {"scale": float("nan")}),
    ({}, {}, {}, {"loss": None}), ({}, {}, {}, {"work": None}), ({}, {}, {}, {"work": A + 4}), ({}, {}, {}, {"bytes": 1000}), ({}, {}, {}, {"sigma": A + 1}), ({}, {}, {}, {"sigma_slow": A}),
    ({}, {}, {}, {"predictor": None}), ({}, {}, {}, {"listed": None})])
def test_predictor_loss_refuses(lib, ctx, pred, samples, grads, change):
    assert _loss(lib, ctx, pred, samples, grads, **change) == lib.ERR_ARG


def test_predictor_loss_refuses_sizes_and_dropouts(lib, ctx):
    assert _loss(lib, ctx, n=1 << 20) == lib.ERR_SHAPE
    assert _loss(lib, ctx, samples={"count": 1 << 31}) == lib.ERR_SHAPE
    assert _loss(lib, None) == lib.ERR_ARG
    assert _loss(lib, ctx, dropout=C.byref(lib.DropoutRule(1.0, 0, 0, None))) == lib.ERR_ARG
    raw, p = lib.raw_library(), _predictor(lib)
    assert raw.mf_predictor_loss_work(ctx, C.byref(p), -1) == lib.ERR_ARG and raw.mf_predictor_loss_work(ctx, None, 5) == lib.ERR_ARG
    assert raw.mf_predictor_loss_work(None, C.byref(p), 5) == lib.ERR_ARG and raw.mf_predictor_loss_work(ctx, C.byref(p), 1 << 31) == lib.ERR_SHAPE


@pytest.mark.parametrize("change", [{"on": None}, {"off": None}, {"count": -1}, {"sigma": None}, {"sigma": A + 2}, {"sigma_slow": A}, {"x_off": None}, {"m": -1}, {"pred": None}])
def test_predict_pairs_refuses(lib, ctx, change):
    a = dict(pred=C.byref(_predictor(lib)), x_on=A, n=5, x_off=A, m=5, on=A, off=A, count=9, sigma=A, sigma_slow=None)
    assert lib.raw_library().mf_predict_pairs(ctx, *{**a, **change}.values()) == lib.ERR_ARG


def test_no_pairs_to_predict(lib, ctx):
    a = [C.byref(_predictor(lib)), None, 0, None, 0, None, None, 0, None, None]
    assert lib.raw_library().mf_predict_pairs(ctx, *a) == lib.OK


def test_structs_match_the_header(lib):
    """Members of the structs these calls take, in order."""
    import re
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "muxmatch.h")).read(), flags=re.S)
    for name, struct in (("mf_predictor", lib.Predictor), ("mf_dropout_rule", lib.DropoutRule), ("mf_samples", lib.Samples), ("mf_gradients", lib.Gradients)):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
        members = [re.search(r"(\w+)$", part.strip()).group(1) for line in body.split(";") if line.strip() for part in line.split(",")]
        assert members == [field for field, _ in struct._fields_], name
