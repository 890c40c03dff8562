"""fp64 oracle of the token operators: norm and rotation, attention, gradients.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

Written from the definitions in include/rtcc.h: one row, one head, one query
at a time over the keys it sees, so that what a query does not see cannot take
part.  Inputs are numpy arrays (any real dtype); everything is computed and
returned in float64.  Beside each result stands the sum of the absolute values
of its terms, from which the tests derive how far rounding may move it.
"""

import numpy as np


# ------------------------------------------------------------- norm, rotation

def _pairs(dim, interleaved):
    p = np.arange(dim // 2)
    return (2 * p, 2 * p + 1) if interleaved else (p, p + dim // 2)


def angles(positions, inv_freq, sections, dim):
    """[rows, dim / 2]: the rotation angle of every pair (0 past the sections)."""
    a = np.zeros((len(positions), dim // 2))
    at = 0
    for axis, n in enumerate(sections):
        f = np.asarray(inv_freq[at:at + n], np.float64)
        a[:, at:at + n] = np.asarray(positions[:, axis], np.float64)[:, None] * f
        at += n
    return a


def rotate(x, angle, interleaved):
    """Rotate the pairs of x [rows, heads, dim] by angle [rows, dim / 2]."""
    i, j = _pairs(x.shape[-1], interleaved)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y = np.empty_like(x)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., i] * s + x[..., j] * c
    return y


def norm_rope(x, weight, angle, eps, interleaved):
    x = np.asarray(x, np.float64)
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if weight is not None:
        n = n * np.asarray(weight, np.float64)
    return rotate(n, angle, interleaved)


def norm_rope_grad(x, weight, angle, eps, interleaved, dy):
    """dx [rows, heads, dim] and dw [heads, dim] (a shared weight's gradient is
    its sum over the heads)."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    g = rotate(dy, -angle, interleaved)
    rms = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x / rms
    gw = g if weight is None else g * np.asarray(weight, np.float64)
    dx = (gw - n * (gw * n).mean(-1, keepdims=True)) / rms
    return dx, (g * n).sum(0)


# ------------------------------------------------------------------ attention

def limits(nq, nk, causal, prefix):
    """Keys that each query sees: the first limits[i]."""
    if not causal:
        return [nk] * nq
    return [min(nk, max(nk - nq + i + 1, min(max(prefix, 0), nk), 0)) for i in range(nq)]


def scores(q, k, place, slope, scale, softcap):
    """Scores of one query against keys k [n, dim], and d score / d (scale q k)."""
    x = scale * (k @ q)
    bend = np.ones_like(x)
    if softcap:
        t = np.tanh(x / softcap)
        x, bend = softcap * t, 1.0 - t * t
    return x - slope * np.abs(place - np.arange(len(k))), bend


class Attention:
    """The forward pass of packed sequences; attributes out, lse, and out_abs =
    sum p |v|.  Rows in no sequence stay NaN.  seqs: (q0, nq, k0, nk, prefix)."""

    def __init__(self, q, k, v, seqs, causal=False, slopes=None, scale=1.0, softcap=0.0):
        self.q, self.k, self.v = (np.asarray(x, np.float64) for x in (q, k, v))
        self.seqs, self.causal, self.scale, self.softcap = seqs, causal, scale, softcap
        heads = self.q.shape[1]
        self.group = heads // self.k.shape[1]
        self.slopes = np.zeros(heads) if slopes is None else np.asarray(slopes, np.float64)
        self.out = np.full(self.q.shape, np.nan)
        self.out_abs = np.zeros(self.q.shape)
        self.lse = np.full((heads, self.q.shape[0]), np.nan)
        for h, row, keys, p, lse, _x, _bend in self.rows():
            v = self.v[keys, h // self.group]
            self.lse[h, row] = lse
            self.out[row, h] = p @ v
            self.out_abs[row, h] = p @ np.abs(v)

    def rows(self):
        """(head, row, its keys' slice, weights, lse, scores, bend) of every row."""
        for q0, nq, k0, nk, prefix in self.seqs:
            for i, n in enumerate(limits(nq, nk, self.causal, prefix)):
                keys = slice(k0, k0 + n)
                for h in range(self.q.shape[1]):
                    x, bend = scores(self.q[q0 + i, h], self.k[keys, h // self.group], nk - nq + i, self.slopes[h],
                                     self.scale, self.softcap)
                    top = x.max() if n else -np.inf
                    if top == -np.inf:
                        p, lse = np.zeros(n), -np.inf
                    else:
                        e = np.exp(x - top)
                        lse = top + np.log(e.sum())
                        p = e / e.sum()
                    yield h, q0 + i, keys, p, lse, x, bend

    def grad(self, dout):
        """dq, dk, dv and, for each, a bound term: the sum of absolute terms with
        every weight's gradient replaced by P (|dP| + |delta| + sum |dout| |out|)
        (what relative errors of P, dP and delta are relative to)."""
        do = np.asarray(dout, np.float64)
        dq, dk, dv = np.zeros(self.q.shape), np.zeros(self.k.shape), np.zeros(self.v.shape)
        bq, bk, bv = np.zeros(self.q.shape), np.zeros(self.k.shape), np.zeros(self.v.shape)
        for h, row, keys, p, _lse, _x, bend in self.rows():
            kh = h // self.group
            k, v, q, g = self.k[keys, kh], self.v[keys, kh], self.q[row, h], do[row, h]
            dp = v @ g
            delta = p @ dp
            ds = p * (dp - delta) * bend * self.scale
            size = p * (np.abs(v) @ np.abs(g) + np.abs(g) @ np.abs(self.out[row, h])) * self.scale
            dq[row, h] = ds @ k
            dk[keys, kh] += np.outer(ds, q)
            dv[keys, kh] += np.outer(p, g)
            bq[row, h] = size @ np.abs(k)
            bk[keys, kh] += np.outer(size, np.abs(q))
            bv[keys, kh] += np.outer(p, np.abs(g))
        return (dq, dk, dv), (bq, bk, bv)
