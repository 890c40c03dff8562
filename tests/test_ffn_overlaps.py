"""Tensors of the feed-forward unit that share memory: refused where a product
would read what another has written.  The refusals stand in the GPU library before
anything is launched, so its workspace functions show them without a GPU; the
addresses are made up and never read."""

import itertools
import random

import pytest

from paper_2608_08330_amd import rtcc as R

ROWS, CHANNELS, HIDDEN, APART = 5, 64, 128, 1 << 20
SAVED = ("gate", "up", "act")
GRADS = ("dx", "dw_gate", "dw_up", "dw_down")


def _forward(saved=True, **kw):
    names = ("x", "w_gate", "w_up", "w_down", "out") + (SAVED if saved else ())
    d = R.rtcc_gated_ffn_desc(abi_version=R.RTCC_ABI_VERSION, precision=R.RTCC_PREC_BF16, rows=ROWS, channels=CHANNELS,
                              hidden=HIDDEN, x_stride=CHANNELS, w_gate_stride=CHANNELS, w_up_stride=CHANNELS,
                              w_down_stride=HIDDEN, out_stride=CHANNELS, hidden_stride=HIDDEN,
                              **{n: (i + 1) * APART for i, n in enumerate(names)})
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _gradients(fwd, want=GRADS, **kw):
    g = R.rtcc_gated_ffn_grad_desc(fwd=fwd, dout=20 * APART, dout_stride=CHANNELS, dx_stride=CHANNELS, dw_gate_stride=CHANNELS,
                                   dw_up_stride=CHANNELS, dw_down_stride=HIDDEN,
                                   **{n: (21 + i) * APART for i, n in enumerate(GRADS) if n in want})
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def _why(call, d):
    """The message of a refusal; None: accepted."""
    try:
        call(d)
    except R.RtccError as e:
        assert e.status == R.RTCC_E_ARG
        return str(e)


def _at(d, name):
    return getattr(d.fwd if hasattr(d, "fwd") and not hasattr(type(d), name) else d, name)


@pytest.mark.parametrize("one,other", [(a, b) for a in SAVED for b in ("x", "w_gate", "w_up", "w_down", "out")]
                         + list(itertools.combinations(SAVED, 2)) + [("out", "w_down")])
def test_forward_refusals(one, other):
    d = _forward()
    assert _why(R.rtcc_gated_ffn_workspace, d) is None
    for shift in (0, 16):
        setattr(d, one, getattr(d, other) + shift)
        why = _why(R.rtcc_gated_ffn_workspace, d)
        assert one in why and other in why and "overlaps" in why
        # the call itself, which ends before a launch as well
        assert _why(lambda x: R.rtcc_gated_ffn(x, 1 << 40, 1 << 40), d) == why


def test_out_may_be_x():
    d = _forward()
    d.out = d.x
    assert _why(R.rtcc_gated_ffn_workspace, d) is None


@pytest.mark.parametrize("one,other", [(a, b) for a in GRADS for b in ("x", "dout", "act", "w_gate", "w_up")]
                         + list(itertools.combinations(GRADS, 2)))
def test_gradient_refusals(one, other):
    g = _gradients(_forward())
    assert _why(R.rtcc_gated_ffn_grad_workspace, g) is None
    for shift in (0, 16):
        setattr(g, one, _at(g, other) + shift)
        why = _why(R.rtcc_gated_ffn_grad_workspace, g)
        assert one in why and other in why and "overlaps" in why
        assert _why(lambda x: R.rtcc_gated_ffn_grad(x, 1 << 40, 1 << 40), g) == why


def test_gradients_in_place_of_what_nothing_reads_any_more():
    """The first product has read dout for dX, and gate, up and w_down; without dX
    the weights of gate and up are not read."""
    for want, one, other in ((("dx",), "dx", "dout"), (("dx",), "dx", "x"), (("dx", "dw_gate", "dw_up"), "dx", "dout"),
                             (("dx", "dw_down"), "dx", "x"), (("dw_gate",), "dw_gate", "w_gate"),
                             (GRADS, "dw_down", "w_down"), (GRADS, "dx", "gate")):
        g = _gradients(_forward(), want)
        setattr(g, one, _at(g, other))
        assert _why(R.rtcc_gated_ffn_grad_workspace, g) is None


def test_no_rows_read_nothing():
    """Weights' gradients of no rows are zeros, wherever the weights lie."""
    g = _gradients(_forward(rows=0))
    g.dw_gate = g.fwd.w_gate
    assert _why(R.rtcc_gated_ffn_grad_workspace, g) is None
    g.dw_up = g.dw_gate
    assert "overlaps" in _why(R.rtcc_gated_ffn_grad_workspace, g)


def test_columns_of_one_buffer_are_apart():
    """gate, up and act as columns of one matrix, and next to each other in turn."""
    d = _forward(hidden_stride=3 * HIDDEN)
    d.up, d.act = d.gate + 2 * HIDDEN, d.gate + 4 * HIDDEN
    assert _why(R.rtcc_gated_ffn_workspace, d) is None
    d.act -= 16
    assert "up overlaps act" in _why(R.rtcc_gated_ffn_workspace, d)


def _bytes(at, rows, stride, width):
    return {at + 2 * (i * stride + j) for i in range(rows) for j in range(width)}


def test_against_the_bytes_themselves():
    """out and act anywhere around each other: contiguous, of equal strides, one row.
    Of two strides with gaps no overlap is found that is none."""
    rng = random.Random(0)
    seen = set()
    for _ in range(3000):
        rows, channels, hidden = rng.choice((1, 2, 7)), 8 * rng.randint(1, 4), 8 * rng.randint(1, 4)
        so, sh = channels + 8 * rng.choice((0, 0, 1, 5)), hidden + 8 * rng.choice((0, 0, 1, 5))
        if rng.random() < 0.4:
            so = sh = max(so, sh)
        d = _forward(rows=rows, channels=channels, hidden=hidden, out_stride=so, hidden_stride=sh, x_stride=channels,
                     w_gate_stride=channels, w_up_stride=channels, w_down_stride=hidden)
        d.out = d.act + 16 * rng.randint(-25, 25)
        shared = bool(_bytes(d.out, rows, so, channels) & _bytes(d.act, rows, sh, hidden))
        why = _why(R.rtcc_gated_ffn_workspace, d)
        exact = rows == 1 or so == sh or so == channels or sh == hidden
        assert why is None or "act overlaps out" in why
        assert (why is not None) == shared if exact else shared or why is None
        seen.add((shared, exact))
    assert len(seen) == 4
