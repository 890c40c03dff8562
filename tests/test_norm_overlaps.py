"""Layer norm: a result is in a tensor's place row by row, or apart from it; what lies
otherwise is refused before a launch (host test library: an accepted call only reports
that there is no GPU)."""

import pytest

from paper_2608_08330_amd import rtcc as R

APART, CHANNELS = 1 << 20, 64


def _norm(**kw):
    names = ("x", "residual", "sum_out", "out")
    d = R.rtcc_layer_norm_desc(abi_version=R.RTCC_ABI_VERSION, precision=R.RTCC_PREC_BF16, rows=5, channels=CHANNELS, eps=1e-5,
                               **{n: (i + 1) * APART for i, n in enumerate(names)},
                               **{n + "_stride": 2 * CHANNELS for n in names})
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _grad(fwd=None, **kw):
    names = ("dout", "dsum", "dx")
    g = R.rtcc_layer_norm_grad_desc(fwd=_norm(**(fwd or {})), dweight=30 * APART, dbias=31 * APART,
                                    **{n: (i + 10) * APART for i, n in enumerate(names)},
                                    **{n + "_stride": 2 * CHANNELS for n in names})
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def _status(call, d, *rest):
    try:
        call(d, *rest, kind="host")
    except R.RtccError as e:
        return e.status, str(e)
    return R.RTCC_OK, ""


@pytest.mark.parametrize("one", ["out", "sum_out"])
@pytest.mark.parametrize("other", ["x", "residual"])
def test_forward(one, other):
    at = getattr(_norm(), other)
    assert _status(R.rtcc_layer_norm, _norm())[0] == R.RTCC_E_STATE
    # in place, and in columns of the same rows
    assert _status(R.rtcc_layer_norm, _norm(**{one: at}))[0] == R.RTCC_E_STATE
    assert _status(R.rtcc_layer_norm, _norm(**{one: at + 2 * CHANNELS}))[0] == R.RTCC_E_STATE
    # a row's part, the next row, another stride
    for kw in ({one: at + 16}, {one: at + 4 * CHANNELS}, {one: at - 4 * CHANNELS}, {one: at, one + "_stride": CHANNELS}):
        status, message = _status(R.rtcc_layer_norm, _norm(**kw))
        assert status == R.RTCC_E_ARG and one in message and other in message
    # one row has no stride
    one_row = {"rows": 1, one: at, one + "_stride": 7}
    assert _status(R.rtcc_layer_norm, _norm(**one_row))[0] == R.RTCC_E_STATE


def test_out_and_sum():
    d = _norm()
    for shift in (0, 16, 4 * CHANNELS):
        status, message = _status(R.rtcc_layer_norm, _norm(sum_out=d.out + shift))
        assert status == R.RTCC_E_ARG and "out" in message
    assert _status(R.rtcc_layer_norm, _norm(sum_out=d.out + 2 * CHANNELS))[0] == R.RTCC_E_STATE


@pytest.mark.parametrize("other", ["dout", "dsum", "sum_out", "x"])
def test_gradient(other):
    fwd = dict(residual=None) if other == "x" else {}
    g = _grad(fwd)
    at = getattr(g, other, None) or getattr(g.fwd, other)
    assert _status(R.rtcc_layer_norm_grad, g, 0, 0)[0] == R.RTCC_E_STATE
    assert _status(R.rtcc_layer_norm_grad, _grad(fwd, dx=at), 0, 0)[0] == R.RTCC_E_STATE
    for kw in (dict(dx=at + 16), dict(dx=at + 4 * CHANNELS), dict(dx=at, dx_stride=CHANNELS)):
        for call, rest in ((R.rtcc_layer_norm_grad, (0, 0)), (R.rtcc_layer_norm_grad_workspace, ())):
            status, message = _status(call, _grad(fwd, **kw), *rest)
            assert status == R.RTCC_E_ARG and "dx" in message and other in message


def test_gradient_reads_no_forward_input_beside_the_normed_tensor():
    """With a residual x and residual are not read: dx may lie anywhere on them."""
    assert _status(R.rtcc_layer_norm_grad, _grad(dx=_norm().x + 16), 0, 0)[0] == R.RTCC_E_STATE


def test_weights_gradients():
    g = _grad()
    for shift, ok in ((0, False), (4, False), (4 * CHANNELS - 4, False), (4 * CHANNELS, True), (-4 * CHANNELS, True)):
        status, message = _status(R.rtcc_layer_norm_grad, _grad(dbias=g.dweight + shift), 0, 0)
        assert status == (R.RTCC_E_STATE if ok else R.RTCC_E_ARG)
        assert ok or "dweight overlaps dbias" in message
    for kw in (dict(dweight=None), dict(dbias=None)):
        assert _status(R.rtcc_layer_norm_grad, _grad(**kw), 0, 0)[0] == R.RTCC_E_STATE
