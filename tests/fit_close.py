"""How near a predictor's gradients are as a whole: the loss evaluated in any precision, and what an evaluation with float32's sums may be off.

`fit_reference` bounds every entry, through every layer, for the worst that roundings can do together, and that is thousands of times what they do.
Here the error of a gradient is one number, its length relative to the gradient's: |g - exact| / |exact|, both over all entries of that parameter."""
import numpy as np

import fit_reference as ref


def evaluate(s, drop=None, scale=None, kind=np.float64, operand=lambda v: v):
    """{name: value} of the loss, predictions and gradients of a problem (as test_gpu_fit's), in arithmetic of type `kind` with the operands of
    every product over samples, features or units rounded by `operand`; and {name: length of the sums of magnitudes}."""
    p = {k: np.asarray(v, dtype=kind) for k, v in s["params"].items()}
    x_on, x_off, on, off = s["x_on"], s["x_off"], s["on"], s["off"]
    count, F, H = len(on), x_on.shape[1], p["b1"].size
    scale = kind(1.0 / max(count, 1) if scale is None else scale)
    real = (on >= 0) & (on < len(x_on)) & (off >= 0) & (off < len(x_off))
    i, j = np.where(real, on, 0), np.where(real, off, 0)

    def times(a, b):
        return operand(a) @ operand(b)

    sides = []
    for x, rows in ((x_on, i), (x_off, j)):
        x = np.asarray(x, dtype=kind)
        if s["eps"] is not None:
            x = x - x.mean(1, keepdims=True)
            x = x / np.sqrt((x * x).mean(1, keepdims=True) + kind(s["eps"]))
        sides.append(x[rows])
    u = np.concatenate(sides, 1)
    x = u * p["ln_w"] + p["ln_b"] if s["eps"] is not None else u
    z1 = times(x, p["W1"].T) + p["b1"]
    if s["sm"] is not None:
        share = np.minimum(np.float32(1.0) - x_on[i, s["sm"][0]], x_off[j, s["sm"][1]]).astype(kind)
        z1 = z1 + np.outer(share, p["W1sm"])
    one = np.ones((1, 1), dtype=kind)
    k1, k2 = (ref.kept(count, H, *drop, layer).astype(kind) for layer in (0, 1)) if drop is not None else (one, one)
    d1 = np.maximum(z1, 0) * k1
    z2 = times(d1, p["W2"].T) + p["b2"]
    d2 = np.maximum(z2, 0) * k2
    out, size, back, total = {}, {}, np.zeros((count, H), dtype=kind), kind(0)
    heads = [("sigma", "W3", "b3", s["target"])] + ([("sigma_slow", "W3slow", "b3slow", s["target_slow"])] if "W3slow" in p else [])
    for name, W, b, t in heads:
        y = 1 / (1 + np.exp(-(d2 @ p[W] + p[b])))
        out[name] = np.where(real, y, 0)
        seen = real & ~np.isnan(t)
        miss = np.where(seen, y - np.where(seen, t, 0).astype(kind), 0)
        total = total + (miss * miss).sum() * scale
        dz = 2 * scale * miss * y * (1 - y)
        out[W], size[W] = dz @ d2, np.abs(dz) @ d2
        out[b], size[b] = dz.sum(keepdims=True), np.abs(dz).sum(keepdims=True)
        back = back + np.outer(dz, p[W])
    out["loss"] = np.array([total])
    dz2 = np.where(z2 > 0, back * k2, 0)
    out["W2"], size["W2"] = times(dz2.T, d1), np.abs(dz2).T @ d1
    out["b2"], size["b2"] = dz2.sum(0), np.abs(dz2).sum(0)
    dz1 = np.where(z1 > 0, times(dz2, p["W2"]) * k1, 0)
    out["b1"], size["b1"] = dz1.sum(0), np.abs(dz1).sum(0)
    if s["sm"] is not None:
        out["W1sm"], size["W1sm"] = share @ dz1, np.abs(share) @ np.abs(dz1)
    out["W1"], size["W1"] = times(dz1.T, x), np.abs(dz1).T @ np.abs(x)
    if s["eps"] is not None:
        dx = dz1 @ p["W1"]
        out["ln_w"], size["ln_w"] = (dx * u).sum(0), np.abs(dx * u).sum(0)
        out["ln_b"], size["ln_b"] = dx.sum(0), np.abs(dx).sum(0)
    return out, size, (z1, z2)


def away_from_kinks(s, drop=None, margin=2e-5):
    """The problem without the samples (they name no pair any more) of which a hidden unit is within `margin` of where its ReLU opens: there a
    rounding, about 1e-6 of what units are sums of, decides whether a gradient passes.  Of 256 units some 1 % of the samples are."""
    z1, z2 = evaluate(s, drop)[2]
    near = (np.abs(z1) < margin).any(1) | (np.abs(z2) < margin).any(1)
    assert near.mean() < 0.2
    return dict(s, on=np.where(near, -1, s["on"]).astype(np.int32))


def room(s, drop=None, scale=None, longest=0):
    """{name: (exact value, |exact|, what |g - exact| / |exact| may be)}.  An evaluation whose products' operands are float32 values to 2^-22 (as two
    fp16 pieces, of which the product of the low ones, 2^-22 again, is left out) and whose sums are float32's: three operand errors of
    2^-22 of every term of a gradient's last sum, 3 (2^-22) of the sums of magnitudes, and through the layers before it what float32's own roundings, of
    2^-24 each, do: three times four as much, and a quarter more for the same in any order, 16 times in all.  Sums one after the other over `longest` terms add
    sqrt(longest) 2^-24 of the magnitudes (errors of either sign), four deviations of it."""
    exact, size, _ = evaluate(s, drop, scale)
    plain = evaluate(s, drop, scale, np.float32)[0]
    out = {}
    for name, value in exact.items():
        length = np.linalg.norm(value)
        away = np.linalg.norm(plain[name].astype(np.float64) - value)
        terms = np.linalg.norm(size[name]) if name in size else length
        out[name] = value, length, (16 * away + (3 * 2.0 ** -22 + 4 * np.sqrt(longest) * 2.0 ** -24 + 2.0 ** -23) * terms) / max(length, 1e-300)
    return out


def distance(got, value):
    return np.linalg.norm(np.asarray(got, dtype=np.float64).reshape(value.shape) - value) / max(np.linalg.norm(value), 1e-300)


def check(got, expected):
    """All of an evaluation against room()."""
    for name, (value, _, most) in expected.items():
        off = distance(got[name], value)
        assert off <= most, f"{name}: off by {off:.3g} of its length, at most {most:.3g}"
