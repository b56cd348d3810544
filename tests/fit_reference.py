"""The definition of the layers and of a predictor's loss in float64, with bounds on what float32 may be off.

Beside every value goes a bound on the error of a float32 evaluation, by running error analysis: a sum of K products
of operands known to errors e is off by at most (K + 2) U sum |products| + sum |operand| e, and so on through the layers.  U is
half a step of float32.  A matrix product may take its operands to OPERAND relative (float32 held as two fp16 pieces).
A ReLU whose input is within its bound of 0 may pass a gradient or not."""
import numpy as np

U = 2.0 ** -24
OPERAND = 2.0 ** -21


def random_bits(seed, step, layer, elements):
    """The 16 random bits of elements 0 .. elements - 1 (Philox 4x32, ten rounds)."""
    u64 = np.uint64
    g = np.arange((elements + 7) // 8, dtype=u64)
    low = u64(0xFFFFFFFF)
    c = [g & low, (g >> u64(32)) | u64(layer << 16), np.full_like(g, step & 0xFFFFFFFF), np.full_like(g, step >> 32)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p0, p1 = u64(0xD2511F53) * c[0], u64(0xCD9E8D57) * c[2]
        c = [(p1 >> u64(32)) ^ c[1] ^ u64(k0), p1 & low, (p0 >> u64(32)) ^ c[3] ^ u64(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = [h for w in c for h in (w & u64(0xFFFF), w >> u64(16))]
    return np.stack(halves, axis=1).reshape(-1)[:elements].astype(np.int64)


def kept(rows, width, p, seed, step, layer):
    """What every element is multiplied by."""
    limit = int(np.rint(np.float64(np.float32(p)) * 65536))
    bits = random_bits(seed, step, layer, rows * width).reshape(rows, width)
    return np.where(bits >= limit, np.float64(np.float32(65536.0 / (65536 - limit))), 0.0)


# additions any value of a row passes through: up to 32 in a lane, six steps over lanes, three over wavefronts, and the division
ROW_SUM = 32 + 6 + 3 + 1


def norm_rows(x, w, b, eps):
    """Layer norm of the rows of x (float64 holding values of the type), and bounds: y, e_y, unit, e_unit, rstd."""
    mean = x.mean(1, keepdims=True)
    d = x - mean
    rstd = 1.0 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    unit = d * rstd
    # the mean is off by ROW_SUM U mean |x|; differences from it by that and a rounding; the variance, relatively, by twice that
    # of the differences and ROW_SUM U; the root halves it
    e_mean = ROW_SUM * U * np.abs(x).mean(1, keepdims=True)
    e_rstd = (ROW_SUM / 2 + 6) * U + (e_mean * rstd) ** 2
    e_unit = np.abs(unit) * (e_rstd + 2 * U) + rstd * e_mean
    y = unit * w + b
    return y, e_unit * np.abs(w) + 2 * U * (np.abs(unit * w) + np.abs(b)), unit, e_unit, rstd, e_rstd


def norm_grad_rows(x, dy, w, eps):
    """dx, dw, db and their bounds."""
    rows = x.shape[0]
    _, _, unit, e_unit, rstd, e_rstd = norm_rows(x, w, 0.0 * w, eps)
    g = dy * w
    mean_g, dot = g.mean(1, keepdims=True), (g * unit).mean(1, keepdims=True)
    e_mean = (ROW_SUM + 1) * U * np.abs(g).mean(1, keepdims=True)
    e_dot = (ROW_SUM + 3) * U * np.abs(g * unit).mean(1, keepdims=True) + (np.abs(g) * e_unit).mean(1, keepdims=True)
    inner = g - mean_g - unit * dot
    e_inner = e_mean + np.abs(unit) * e_dot + e_unit * np.abs(dot) + 4 * U * (np.abs(g) + np.abs(mean_g) + np.abs(unit * dot))
    dx, e_dx = rstd * inner, rstd * (e_inner + np.abs(inner) * (e_rstd + 2 * U))
    # rows of a thread, groups of lanes, slices of workgroups (their numbers are at most these)
    steps = max(8, rows // 256) + 64 + 64 + 16
    dw, e_dw = (dy * unit).sum(0), steps * U * np.abs(dy * unit).sum(0) + (np.abs(dy) * e_unit).sum(0)
    return dx, e_dx, dw, e_dw, dy.sum(0), steps * U * np.abs(dy).sum(0)


def product(A, e_A, B, e_B):
    """A @ B with its bound."""
    K = A.shape[1]
    e_A, e_B = e_A + OPERAND * np.abs(A), e_B + OPERAND * np.abs(B)
    return A @ B, (K + 2) * U * (np.abs(A) @ np.abs(B)) + e_A @ np.abs(B) + np.abs(A) @ e_B + e_A @ e_B


def loss(params, x_on, x_off, on, off, target, scale, target_slow=None, drop=None, sm=None, eps=None):
    """Loss, predictions and gradients with bounds: {name: (value, bound)}, names as in a predictor's dictionary besides
    "loss", "sigma" and "sigma_slow"."""
    p = {k: np.asarray(v, dtype=np.float64) for k, v in params.items()}
    n, m, F, H = len(x_on), len(x_off), x_on.shape[1], p["b1"].size
    real = (on >= 0) & (on < n) & (off >= 0) & (off < m)
    i, j = np.where(real, on, 0), np.where(real, off, 0)
    count = len(on)
    sides = []
    for x, rows, part in ((x_on, i, slice(0, F)), (x_off, j, slice(F, 2 * F))):
        x = np.asarray(x, dtype=np.float64)
        if eps is not None:
            _, _, unit, e_unit, _, _ = norm_rows(x, p["ln_w"][part], p["ln_b"][part], eps)
            sides.append((unit[rows], e_unit[rows]))
        else:
            sides.append((x[rows], np.zeros((count, F))))
    unit, e_unit = np.concatenate([s[0] for s in sides], 1), np.concatenate([s[1] for s in sides], 1)
    gain, beta = (p["ln_w"], p["ln_b"]) if eps is not None else (np.ones(2 * F), np.zeros(2 * F))
    # layer 1 with the norm folded in: weights off by a rounding, the bias by those of its sum
    W, e_W = p["W1"] * gain, U * np.abs(p["W1"] * gain)
    b, e_b = p["b1"] + p["W1"] @ beta, (2 * F + 2) * U * (np.abs(p["W1"]) @ np.abs(beta) + np.abs(p["b1"]))
    z1, e_z1 = product(unit, e_unit, W.T, e_W.T)
    z1, e_z1 = z1 + b, e_z1 + e_b + 2 * U * (np.abs(z1) + np.abs(b))
    share = None
    if sm is not None:
        share = np.minimum(np.float32(1.0) - x_on[i, sm[0]], x_off[j, sm[1]]).astype(np.float64)
        z1 = z1 + np.outer(share, p["W1sm"])
        e_z1 = e_z1 + 2 * U * (np.abs(np.outer(share, p["W1sm"])) + np.abs(z1))
    one = np.ones((count, H))
    k1, k2 = (kept(count, H, *drop, layer) for layer in (0, 1)) if drop is not None else (one, one)
    d1, e_d1 = np.maximum(z1, 0) * k1, e_z1 * k1 + 2 * U * np.abs(np.maximum(z1, 0) * k1)
    z2, e_z2 = product(d1, e_d1, p["W2"].T, np.zeros((H, H)))
    z2, e_z2 = z2 + p["b2"], e_z2 + 2 * U * (np.abs(z2) + np.abs(p["b2"]))
    d2, e_d2 = np.maximum(z2, 0) * k2, e_z2 * k2 + 2 * U * np.abs(np.maximum(z2, 0) * k2)
    out, heads = {}, [("sigma", "W3", "b3", target)]
    if "W3slow" in p:
        heads.append(("sigma_slow", "W3slow", "b3slow", target_slow))
    # samples that a weight's gradient passes through one after the other (a workgroup's, then slices of workgroups)
    steps = count / 64 + 64 + 32 + 64
    back, e_back, total, e_total = np.zeros((count, H)), np.zeros((count, H)), 0.0, 0.0
    for name, Wn, bn, t in heads:
        z = d2 @ p[Wn] + p[bn]
        e_z = (H + 4) * U * (np.abs(d2) @ np.abs(p[Wn]) + np.abs(p[bn])) + e_d2 @ np.abs(p[Wn])
        y = 1.0 / (1.0 + np.exp(-z))
        e_y = y * (1 - y) * e_z * 1.01 + 8 * U * y          # an exponential (2 steps), an addition and a division
        out[name] = np.where(real, y, 0.0), np.where(real, e_y, 0.0)
        if t is None:
            continue
        seen = real & ~np.isnan(t)
        miss = np.where(seen, y - np.where(seen, t, 0.0), 0.0)
        e_miss = np.where(seen, e_y + U * np.abs(miss), 0.0)
        total += (miss ** 2).sum() * scale
        e_total += scale * ((2 * np.abs(miss) * e_miss + e_miss ** 2).sum() + steps * U * (miss ** 2).sum())
        slope = y * (1 - y)
        dz = 2 * scale * miss * slope
        e_dz = np.where(seen, 2 * scale * (e_miss * slope + np.abs(miss) * (e_y + U)) + 6 * U * np.abs(dz), 0.0)
        out[Wn] = dz @ d2, steps * U * (np.abs(dz) @ np.abs(d2)) + e_dz @ np.abs(d2) + np.abs(dz) @ e_d2 + e_dz @ e_d2
        out[bn] = np.array([dz.sum()]), np.array([steps * U * np.abs(dz).sum() + e_dz.sum()])
        back += np.outer(dz, p[Wn])
        e_back += np.outer(e_dz, np.abs(p[Wn])) + 3 * U * np.abs(np.outer(dz, p[Wn]))
    out["loss"] = np.array([total]), np.array([e_total + 4 * U * total])
    if target is None:
        return out

    def masked(v, e_v, z, e_z, k):
        """Back through dropout and ReLU."""
        doubt = np.abs(z) <= e_z
        v, e_v = v * k, e_v * k + 2 * U * np.abs(v * k)
        return np.where(z > 0, v, 0.0), np.where(doubt, np.abs(v) + e_v, np.where(z > 0, e_v, 0.0))

    def summed(A, e_A, B, e_B):
        """A^T B over samples."""
        e_A, e_B = e_A + OPERAND * np.abs(A), e_B + OPERAND * np.abs(B)
        return A.T @ B, steps * U * (np.abs(A).T @ np.abs(B)) + e_A.T @ np.abs(B) + np.abs(A).T @ e_B + e_A.T @ e_B

    dz2, e_dz2 = masked(back, e_back, z2, e_z2, k2)
    out["W2"] = summed(dz2, e_dz2, d1, e_d1)
    out["b2"] = dz2.sum(0), steps * U * np.abs(dz2).sum(0) + e_dz2.sum(0)
    dz1, e_dz1 = masked(*product(dz2, e_dz2, p["W2"], np.zeros((H, H))), z1, e_z1, k1)
    h, e_h = dz1.sum(0), steps * U * np.abs(dz1).sum(0) + e_dz1.sum(0)
    out["b1"] = h, e_h
    if sm is not None:
        out["W1sm"] = share @ dz1, steps * U * (np.abs(share) @ np.abs(dz1)) + np.abs(share) @ e_dz1
    G, e_G = summed(dz1, e_dz1, unit, e_unit)
    out["W1"] = G * gain + np.outer(h, beta), e_G * np.abs(gain) + np.outer(e_h, np.abs(beta)) + 4 * U * (np.abs(G * gain) + np.abs(np.outer(h, beta)))
    if eps is not None:
        out["ln_w"] = (p["W1"] * G).sum(0), (np.abs(p["W1"]) * (e_G + (H + 2) * U * np.abs(G))).sum(0)
        out["ln_b"] = h @ p["W1"], (e_h + (H + 2) * U * np.abs(h)) @ np.abs(p["W1"])
    return out


def within(got, value, bound, what, least=0.0):
    """Every entry within its bound and half a step of its type: `least` relative, but below float16's smallest normal number,
    2^-14, its steps are all 2^-24 (10 fraction bits below 2^-14), so half of one is 2^-25 there, more than 2^-11 of the value."""
    got = np.asarray(got, dtype=np.float64).reshape(np.shape(value))
    off, room = np.abs(got - value), bound + least * (np.abs(value) + bound) + (2.0 ** -25 if least == 2.0 ** -11 else 2.0 ** -149)
    worst = np.unravel_index(np.argmax(off - room), np.shape(off)) if off.size else None
    assert off.size == 0 or (off <= room).all(), f"{what}{worst}: {got[worst]!r}, expected {value[worst]!r} within {room[worst]:.3g}"
