"""fp64 oracle of the operators around the attention: layer norm of a residual
stream, the gated feed-forward unit, and their gradients.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

Written from the definitions in include/rtcc.h.  Inputs are numpy arrays (any
real dtype); everything is computed and returned in float64.  Beside the results
stand the sums of the absolute values of their terms, from which the tests derive
how far rounding may move them.
"""

import numpy as np
from scipy import special


def f64(x):
    return np.asarray(x, np.float64)


# ----------------------------------------------------------------- layer norm

def layer_norm(x, residual, weight, bias, eps):
    """out, sum, and the normed values n with r = 1 / sqrt(var + eps)."""
    s = f64(x) if residual is None else f64(x) + f64(residual)
    d = s - s.mean(1, keepdims=True)
    r = 1.0 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    out = d * r
    if weight is not None:
        out = out * f64(weight)
    if bias is not None:
        out = out + f64(bias)
    return out, s, d * r, r


def layer_norm_grad(s, weight, eps, dout, dsum):
    """dx, dweight, dbias of the norm of s."""
    _, _, n, r = layer_norm(s, None, None, None, eps)
    dy = f64(dout)
    g = dy if weight is None else dy * f64(weight)
    dx = r * (g - g.mean(1, keepdims=True) - n * (g * n).mean(1, keepdims=True))
    if dsum is not None:
        dx = dx + f64(dsum)
    return dx, (dy * n).sum(0), dy.sum(0)


# ---------------------------------------------------------- gated feed-forward

def activation(z, gelu):
    """Values and slopes."""
    if gelu:
        phi = special.ndtr(z)
        return z * phi, phi + z * np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
    s = special.expit(z)
    return z * s, s * (1 + z * (1 - s))


def gated_ffn(x, w_gate, w_up, w_down, gelu):
    """out, g, u, h."""
    g, u = f64(x) @ f64(w_gate).T, f64(x) @ f64(w_up).T
    h = activation(g, gelu)[0] * u
    return h @ f64(w_down).T, g, u, h


def gated_ffn_grad(x, w_gate, w_up, w_down, gelu, gate, up, act, dout):
    """dx, dw_gate, dw_up, dw_down, and the inner dg, du, dh, of a forward call
    that stored gate, up and act."""
    a, slope = activation(f64(gate), gelu)
    dy = f64(dout)
    dh = dy @ f64(w_down)
    du, dg = dh * a, dh * f64(up) * slope
    return (dg @ f64(w_gate) + du @ f64(w_up), dg.T @ f64(x), du.T @ f64(x), dy.T @ f64(act)), (dg, du, dh)
