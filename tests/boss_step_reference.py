"""Plain restatement (NumPy) of linear layers, layer normalisation and AdamW, with the sums of absolute terms that error bounds are stated in.
Test infrastructure; shares nothing with the CUDA library."""
import math

import numpy as np
from scipy.special import erf

import boss_reference as R


def act(z, name):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + erf(z / math.sqrt(2.0)))
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    return z


def act_slope(z, name):
    if name == "relu":
        return (z > 0).astype(float)
    if name == "gelu":
        return 0.5 * (1.0 + erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1.0 - s)
    return np.ones_like(z)


def linear(x, w, bias, name, residual):
    """out, pre, and the sum of absolute terms of pre."""
    z = x @ w.T + (0.0 if bias is None else bias)
    size = np.abs(x) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    return act(z, name) + (0.0 if residual is None else residual), z, size


def linear_grad(x, w, dout, name, pre, residual):
    g = dout * (1.0 if name is None else act_slope(pre, name))
    got = {"dx": g @ w + (0.0 if residual is None else residual), "dw": g.T @ x, "dbias": g.sum(0)}
    size = {"dx": np.abs(g) @ np.abs(w), "dw": np.abs(g).T @ np.abs(x), "dbias": np.abs(g).sum(0)}
    return got, size, g


def layer_norm(x, gamma, beta, eps):
    c = x - x.mean(1, keepdims=True)
    r = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    h = c * r
    return h * (1.0 if gamma is None else gamma) + (0.0 if beta is None else beta), h, r


def layer_norm_grad(x, gamma, eps, dout, residual):
    _, h, r = layer_norm(x, None, None, eps)
    g = dout * (1.0 if gamma is None else gamma)
    dx = r * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True)) + (0.0 if residual is None else residual)
    return {"dx": dx, "dgamma": (dout * h).sum(0), "dbeta": dout.sum(0)}, h, r, g


# ---------------------------------------------------------------------------------------------------------------- AdamW

def adamw(p, g, m, v, rule, decay, scale=None):
    """One step in the type of the arrays (float64, or float32 with every operation rounded by itself); rule: lr, beta1, beta2, eps, t (this step's)."""
    f = p.dtype.type
    if scale is not None:
        g = g * f(scale)
    m = m * f(rule["beta1"]) + g * f(1.0 - rule["beta1"])
    v = v * f(rule["beta2"]) + (g * g) * f(1.0 - rule["beta2"])
    den = np.sqrt(v * f(1.0 / (1.0 - rule["beta2"] ** rule["t"]))) + f(rule["eps"])
    p = p * f(1.0 - rule["lr"] * decay) - (m / den) * f(rule["lr"] / (1.0 - rule["beta1"] ** rule["t"]))
    return p, m, v


def draws(n, seed, tensor, t):
    """Two 16-bit draws for each of n elements."""
    blocks = np.arange((n + 3) // 4)
    w = R.philox(blocks & 0xFFFFFFFF, tensor, t & 0xFFFFFFFF, t >> 32, seed & 0xFFFFFFFF, seed >> 32)
    w = np.stack([x.astype(np.int64) for x in w], 1).reshape(-1)[:n]
    return w & 0xFFFF, w >> 16


def e4m3_values():
    """Every byte's number (nan for the two codes that are none)."""
    b = np.arange(256)
    e, f = (b >> 3) & 15, b & 7
    x = np.where(e == 0, f * 2.0**-9, (8 + f) * 2.0 ** (e.astype(float) - 10))
    x = np.where((b & 127) == 127, np.nan, x)
    return np.where(b > 127, -x, x)


def to_codes(x, u, root):
    """Moments of one tensor (their unrounded values in float32) -> codes' values in units, scale bytes, magnitudes in units, steps there."""
    f = np.float32
    n = len(x)
    pad = np.zeros((n + 255) // 256 * 256, dtype=f)
    pad[:n] = np.abs(x)
    top = pad.reshape(-1, 256).max(1)
    byte = np.where(top > 0, np.maximum(np.frexp(top)[1] - 1 + 127 - 7, 1), 0)
    units = np.abs(x) / np.repeat(np.where(byte > 0, 2.0 ** (byte - 127.0), 1.0), 256)[:n]
    step = 2.0 ** (np.floor(np.log2(np.maximum(units, 2.0**-6))) - 3)
    # numbers below 2^-6 are added to it in fp32 before their lower neighbour is looked for
    at = np.where(units < 2.0**-6, (f(2.0**-6) + units.astype(f)).astype(float) - 2.0**-6, units)
    if root:
        lo = np.floor(at / step) * step
        a, lo32, hi32 = units.astype(f), lo.astype(f), (lo + step).astype(f)
        up = (a - lo32) * (a + lo32) > u.astype(f) * f(2.0**-16) * ((hi32 - lo32) * (hi32 + lo32))
        code = np.where(up, lo + step, lo)
        code = np.where((x > 0) & (code == 0), 2.0**-9, code)
    else:
        code = np.floor(at / step + u / 65536.0) * step
    return code * np.sign(x), byte.astype(np.uint8), units, step
