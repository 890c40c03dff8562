"""Layer norm of rows whose mean is far larger than their spread.

With U = 2^-24: a row's sum takes at most 47 roundings on the way from a value to the
total (32 values a thread, 6 exchanges of lanes, 8 waves, the division), so the first
mean is off by e <= 47 U |mean|, 47 steps of the values' last bit.  Differences from it
are exact where the row's values lie within a factor of two of each other, and so are
sums of equal ones: up to 2^14 times 47 steps is below 2^24 of them.  What is left of
the mean is then known to the precision of the differences and not of the values."""

import numpy as np
import pytest

from oracle import blocks as O
from paper_2608_08330_amd import rtcc as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# every number of threads a row
CHANNELS = [8, 72, 384, 1000, 2040, 4104, 8200, 16384]
VALUES = [1000.1, -77777.77, 0.1, 3.0e6 + 0.25]


def _run(x, w, b, eps, dy=None, residual=None):
    """out, and with dy the gradients dx, dweight, dbias."""
    import torch
    out = torch.empty_like(x)
    total = None if residual is None else torch.empty_like(x)
    d = R.layer_norm_desc(x, out, w, b, residual=residual, sum_out=total, eps=eps)
    R.rtcc_layer_norm(d)
    if dy is None:
        torch.cuda.synchronize()
        return out
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    g = R.layer_norm_grad_desc(d, dy, dx, dweight=dw, dbias=db)
    n = R.rtcc_layer_norm_grad_workspace(g)
    space = torch.empty(n, dtype=torch.uint8, device="cuda")
    R.rtcc_layer_norm_grad(g, space.data_ptr(), n)
    torch.cuda.synchronize()
    return out, dx, dw, db


def _weights(channels, gen):
    import torch
    return [t.cuda() for t in (1 + 0.2 * torch.randn(channels, generator=gen), 0.3 * torch.randn(channels, generator=gen))]


@pytest.mark.parametrize("channels", CHANNELS)
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_rows_of_one_value_are_the_bias(channels, eps):
    """Whatever the value and eps: the differences are exactly zero."""
    import torch
    gen = torch.Generator().manual_seed(channels)
    w, b = _weights(channels, gen)
    rows = len(VALUES) * 3
    x = torch.tensor(VALUES * 3, dtype=torch.float32, device="cuda")[:, None].expand(rows, channels).contiguous()
    dy = torch.randn(rows, channels, generator=gen).cuda()
    out, _dx, dw, _db = _run(x, w, b, eps, dy)
    assert torch.equal(out, b.expand(rows, channels))
    assert not dw.any()


@pytest.mark.parametrize("channels", CHANNELS)
def test_bf16_sums_of_one_value_are_the_bias(channels):
    """bf16 rows whose float32 sums have more bits than a mean keeps."""
    import torch
    w, b = _weights(channels, torch.Generator().manual_seed(1))
    x, r = (torch.full((5, channels), v, dtype=torch.bfloat16, device="cuda") for v in (1000.0, 0.0041))
    assert torch.equal(_run(x, w, b, 1e-12, residual=r), b.bfloat16().expand(5, channels))


@pytest.mark.parametrize("channels", CHANNELS[1:])
@pytest.mark.parametrize("shift,spread", [(2000.0, 0.01), (-50000.0, 0.5), (3.0, 3e-5)])
def test_rows_far_from_zero(channels, shift, spread):
    """Like rows around zero of the same differences t = x - shift, which float64
    holds exactly.  A difference from the first mean is exact and at most |t - mean| + e,
    one from the second mean carries (46 + 2) U of their mean and a rounding; the
    variance twice that and its own sums.  n has r times the first, and rel |n|."""
    import torch
    gen = torch.Generator().manual_seed(channels)
    w, b = _weights(channels, gen)
    rows, eps = 40, 1e-12
    x = (torch.randn(rows, channels, generator=gen).clamp(-6, 6) * spread + shift).cuda()
    dy = torch.randn(rows, channels, generator=gen).cuda()
    got = [t.double().cpu().numpy() for t in _run(x, w, b, eps, dy)]
    x, dy, w, b = (t.double().cpu().numpy() for t in (x, dy, w, b))
    t = x - shift
    y, _, n, r = O.layer_norm(t, None, w, b, eps)
    e = 47 * U * np.abs(x).mean(1, keepdims=True)
    d = np.abs(t - t.mean(1, keepdims=True)) + e  # the differences as the kernel holds them
    slip = 48 * U * d.mean(1, keepdims=True) + 2 * U * d
    square = 1 / (r * r)  # variance and eps
    # the sum of squares is of d, from which the square of what is left of the mean (at
    # most e) is taken: both are held to their own size
    rel = (48 * U * ((d * d).mean(1, keepdims=True) + e * e) + 2 * (slip * d).mean(1, keepdims=True)) / square + 4 * U
    en = slip * r + rel * np.abs(n)
    assert (np.abs(got[0] - y) <= en * np.abs(w) + 4 * U * (np.abs(n * w) + np.abs(b) + np.abs(y))).all()

    ex, ew, eb = O.layer_norm_grad(t, w, eps, dy, None)
    gw = np.abs(dy * w)
    dots = (gw * np.abs(n)).mean(1, keepdims=True)
    terms = gw + gw.mean(1, keepdims=True) + np.abs(n) * dots
    slack = r * ((48 * U + rel) * terms + en * dots + np.abs(n) * (gw * en).mean(1, keepdims=True))
    assert (np.abs(got[1] - ex) <= 1.01 * slack + 4 * U * np.abs(ex)).all()  # 1.01: products of two errors
    many = (rows + 8) * U
    assert (np.abs(got[2] - ew) <= many * (np.abs(dy * n)).sum(0) + np.abs(dy * en).sum(0)).all()
    assert (np.abs(got[3] - eb) <= many * np.abs(dy).sum(0)).all()
