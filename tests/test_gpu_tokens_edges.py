"""GPU token operators at the edges of their descriptions: buffers of exactly
the stated size, sizes and places near the limits, caps of every size.

Tolerances as in test_gpu_tokens.py: U and B are one rounding to float32 and
bf16; each test says what it adds."""

import numpy as np
import pytest

from oracle import tokens as T
from paper_2608_08330_amd import rtcc as R
from tests.test_gpu_tokens import B, PRECISIONS, U, Case, Rope, _f64, _workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("precision", PRECISIONS)
def test_gradient_of_an_absent_weight_is_one_row(precision):
    """Without a weight its gradient has head_dim values, whatever the flag for
    weights of every head says: what lies behind them is not written."""
    import torch
    rows, heads, dim = 90, (5, 3), 48
    c = Rope(precision, rows, *heads, dim, (8, 8, 8), False, weights="none")
    dy = [g.cuda() for g in c.dy]
    dx = [torch.empty_like(g) for g in dy]
    dw = [torch.full((h, dim), 7.0, device="cuda") for h in heads]
    g = R.norm_rope_grad_desc(c.desc(c.gx), dy[0], dy[1], dx[0], dx[1], dw[0][0], dw[1][0])
    g.fwd.q_weight_per_head = g.fwd.k_weight_per_head = 1
    n = R.rtcc_norm_rope_grad_workspace(g)
    space = _workspace(n)
    R.rtcc_norm_rope_grad(g, space.data_ptr(), n)
    torch.cuda.synchronize()
    for i in range(2):
        assert (dw[i][1:] == 7.0).all()
        want = T.norm_rope_grad(_f64(c.x[i]), None, c.angle, c.eps, False, _f64(c.dy[i]))[1].sum(0)
        x = _f64(c.x[i])
        # terms g x r: |g| of a pair's length, rms-normed x
        size = (np.linalg.norm(_f64(c.dy[i]), axis=-1, keepdims=True) * np.abs(x) /
                np.sqrt((x * x).mean(-1, keepdims=True) + c.eps)).sum((0, 1))
        assert (np.abs(_f64(dw[i][0]) - want) <= (dim + 64 + 2 * np.sqrt(rows * heads[i])) * U * size).all()
