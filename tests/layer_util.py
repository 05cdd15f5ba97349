"""The radial network's hidden layers in float64 (numpy), and how far a call may be from them.

The bounds count, element by element, what each step may lose (u = 2^-24 is half a step of float32 relative to the value, 2 u where the
tensor cores cut off instead of rounding; half = finfo(type).eps / 2):

  products   float32 factors are three bfloat16 each, and the three of nine term products that are left out are
             below 2 * 2^-22 + 2^-30 of the product: 9 u of the sum of magnitudes.  A gradient of a bfloat16 layer is two terms, the second
             rounded to 8 bits: 2^-16 of it (256 u).  A chain of n additions loses at most 2 u of the sum of magnitudes each
             time; a contraction of K makes K / 16 additions to each of two accumulators (the second, of five terms, holds
             2^-6 of the magnitudes), which are added: 2 (K / 16 + 1) u + 10 (K / 16) 2^-6 u + u, below (2.2 K / 16 + 4) u.  With one or two
             bfloat16 terms up to 2 K / 16 additions: 4 K / 16 + 2.  Sums over rows: chains of 16, then groups and
             shares added one after another, rounding: at most 36 + rows / 64 + 600 additions' u.
  activation the fast exponential is within 2 steps and |z| u, the division within 2 steps, root and others less: 24 u of max(|z|, 1);
             erff, tanhf: 2 steps of a value up to 1, times |z|.  Slopes: the same, below 32 u (1 + |z|).
             Slopes of the activations are below 1.13, second derivatives below 1.2 (silu 0.5, tanh 0.77, gelu 0.8).
"""
import numpy as np

U = 2.0 ** -24
ACTS = {"none": 0, "silu": 1, "tanh": 2, "gelu": 3}


def erf(z):
    import torch
    return torch.erf(torch.from_numpy(np.ascontiguousarray(z))).numpy()


def act(z, name):
    if name == "silu":
        return z * (0.5 + 0.5 * np.tanh(0.5 * z))
    if name == "tanh":
        return np.tanh(z)
    if name == "gelu":
        return 0.5 * z * (1 + erf(z / np.sqrt(2.0)))
    return z


def slope(z, name):
    if name == "silu":
        s = 0.5 + 0.5 * np.tanh(0.5 * z)
        return s + z * s * (1 - s)
    if name == "tanh":
        return 1 - np.tanh(z) ** 2
    if name == "gelu":
        return 0.5 * (1 + erf(z / np.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
    return np.ones_like(z)


def act_error(z, name):
    return 0.0 if name == "none" else 24 * U * np.maximum(np.abs(z), 1)


def slope_error(z, name):
    return 0.0 if name == "none" else 32 * U * (1 + np.abs(z))


def chain(k, float32):
    """Steps of u that a contraction of k may lose, of the sum of magnitudes."""
    return 9 + 2.2 * (k / 16 + 1) + 4 if float32 else 4 * (k / 16 + 1) + 2


def linear_fwd(x, W, b, r, name, half):
    """(y, bound): float64 arrays of the real rows."""
    float32 = half < 2.0 ** -20
    z = x @ W + (0 if b is None else b)
    magnitude = np.abs(x) @ np.abs(W) + (0 if b is None else np.abs(b))
    err = 1.13 * (chain(x.shape[1], float32) + 2) * U * magnitude + act_error(z, name)
    y = act(z, name) + (0 if r is None else r)
    if r is not None:
        err = err + U * np.abs(y)
    return y, err * (1 + 2 * half) + half * np.abs(y) + 1e-37


def linear_bwd(x, W, b, g, name, half):
    """((grad_x, grad_W, grad_b), bounds)"""
    float32 = half < 2.0 ** -20
    z = x @ W + (0 if b is None else b)
    magnitude = np.abs(x) @ np.abs(W) + (0 if b is None else np.abs(b))
    gz = g * slope(z, name)
    ez = 0.0 if name == "none" else 1.2 * (chain(x.shape[1], float32) + 2) * U * magnitude
    e_gz = np.abs(g) * (ez + slope_error(z, name)) + U * np.abs(gz)
    terms = 0 if float32 or name == "none" else 256
    rows = x.shape[0]
    gx, gW, gb = gz @ W.T, x.T @ gz, gz.sum(0)
    e_x = e_gz @ np.abs(W).T + (chain(W.shape[1], float32) + terms) * U * (np.abs(gz) @ np.abs(W).T)
    sums = 36 + rows / 64 + 600
    e_W = np.abs(x).T @ e_gz + (sums + 9 + terms) * U * (np.abs(x).T @ np.abs(gz))
    e_b = e_gz.sum(0) + sums * U * np.abs(gz).sum(0)
    return (gx, gW, gb), tuple(e * (1 + 2 * half) + half * np.abs(v) + 1e-37 for v, e in ((gx, e_x), (gW, e_W), (gb, e_b)))


def _norm(x, eps):
    """xh, 1 / sqrt(variance + eps) and bounds of xh: the mean loses (n + 2) u of the mean magnitude, differences u, the
    variance (n + 4) u of itself and twice the mean's error, root and division 2 u more."""
    n = x.shape[1]
    mean = x.mean(1, keepdims=True)
    d = x - mean
    var = (d * d).mean(1, keepdims=True)
    inv = 1 / np.sqrt(var + eps)
    e_mean = (n + 2) * U * np.abs(x).mean(1, keepdims=True)
    e_d = e_mean + U * np.abs(d)
    e_var = 2 * (np.abs(d) * e_d).mean(1, keepdims=True) + (n + 4) * U * var
    rel = 0.5 * e_var / (var + eps) + 4 * U
    xh = d * inv
    return xh, inv, e_d * inv + rel * np.abs(xh) + 2 * U * np.abs(xh), rel


def norm_fwd(x, w, c, eps, name, half):
    xh, _, e, _ = _norm(x, eps)
    z = xh * w + c
    err = 1.13 * (e * np.abs(w) + 2 * U * (np.abs(xh * w) + np.abs(c))) + act_error(z, name)
    y = act(z, name)
    return y, err * (1 + 2 * half) + half * np.abs(y) + 1e-37


def norm_bwd(x, w, c, g, eps, name, half):
    n, rows = x.shape[1], x.shape[0]
    xh, inv, e, rel = _norm(x, eps)
    z = xh * w + c
    gz = g * slope(z, name)
    ez = 0.0 if name == "none" else 1.2 * (e * np.abs(w) + 2 * U * (np.abs(xh * w) + np.abs(c)))
    e_gz = np.abs(g) * (ez + slope_error(z, name)) + U * np.abs(gz)
    u = gz * w
    e_u = e_gz * np.abs(w) + U * np.abs(u)
    m0, m1 = u.mean(1, keepdims=True), (u * xh).mean(1, keepdims=True)
    e0 = e_u.mean(1, keepdims=True) + (n + 2) * U * np.abs(u).mean(1, keepdims=True)
    e1 = (e_u * np.abs(xh) + np.abs(u) * e).mean(1, keepdims=True) + (n + 3) * U * np.abs(u * xh).mean(1, keepdims=True)
    inner = u - m0 - xh * m1
    gx = inner * inv
    e_x = (e_u + e0 + np.abs(xh) * e1 + e * np.abs(m1) + 3 * U * (np.abs(u) + np.abs(m0) + np.abs(xh * m1))) * inv + (rel + 2 * U) * np.abs(gx)
    sums = rows / 8 + 700
    gw, gc = (gz * xh).sum(0), gz.sum(0)
    e_w = (e_gz * np.abs(xh) + np.abs(gz) * e).sum(0) + sums * U * np.abs(gz * xh).sum(0)
    e_c = e_gz.sum(0) + sums * U * np.abs(gz).sum(0)
    return (gx, gw, gc), tuple(e * (1 + 2 * half) + half * np.abs(v) + 1e-37 for v, e in ((gx, e_x), (gw, e_w), (gc, e_c)))


def assert_within(got, want, bound, what=""):
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - want) - bound
    if over.size:
        i = np.unravel_index(np.argmax(over), over.shape)
        assert over[i] <= 0, f"{what}{list(map(int, i))}: {got[i]} for {want[i]}, off {abs(got[i] - want[i]):.3g}, bound {np.broadcast_to(bound, want.shape)[i]:.3g}"
