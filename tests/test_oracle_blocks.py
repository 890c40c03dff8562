"""The oracle of layer norm and the gated feed-forward unit against differences
and against library routines, and what the operators and their descriptions
refuse (host test library: the checks are the GPU library's, the launchers only
report that there is no GPU)."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import blocks as O
from paper_2608_08330_amd import rtcc as R


# --------------------------------------------------------------------- oracle

def _differences(f, args, grads, h=1e-5):
    """Central differences of f, with an error of order h^2 = 1e-10."""
    for which, grad in enumerate(grads):
        for at in list(np.ndindex(*args[which].shape))[::2]:
            lo, hi = [a.copy() for a in args], [a.copy() for a in args]
            lo[which][at] -= h
            hi[which][at] += h
            assert abs((f(*hi) - f(*lo)) / (2 * h) - grad[at]) < 1e-8


def test_layer_norm_gradient_against_differences():
    rng = np.random.default_rng(0)
    x, w, b, dy, ds = (rng.normal(size=s) for s in ((3, 16), (16,), (16,), (3, 16), (3, 16)))

    def loss(x, w, b):
        out, s, _, _ = O.layer_norm(x, None, w, b, 1e-2)
        return (out * dy).sum() + (s * ds).sum()

    _differences(loss, [x, w, b], O.layer_norm_grad(x, w, 1e-2, dy, ds))


@pytest.mark.parametrize("gelu", [False, True])
def test_gated_ffn_gradient_against_differences(gelu):
    rng = np.random.default_rng(1)
    args = [rng.normal(size=s) for s in ((3, 8), (16, 8), (16, 8), (8, 16))]
    dy = rng.normal(size=(3, 8))
    _, g, u, h = O.gated_ffn(*args, gelu)
    grads, _ = O.gated_ffn_grad(*args, gelu, g, u, h, dy)
    _differences(lambda *a: (O.gated_ffn(*a, gelu)[0] * dy).sum(), args, grads)


def test_oracle_against_library():
    rng = np.random.default_rng(2)
    x, r, w, b = (torch.from_numpy(rng.normal(size=s)) for s in ((5, 24), (5, 24), (24,), (24,)))
    out, s, _, _ = O.layer_norm(x, r, w, b, 1e-5)
    assert np.abs(out - torch.nn.functional.layer_norm(x + r, (24,), w, b, 1e-5).numpy()).max() < 1e-12
    z = torch.linspace(-9, 9, 101, dtype=torch.float64)
    assert np.abs(O.activation(z.numpy(), False)[0] - torch.nn.functional.silu(z).numpy()).max() < 1e-14
    assert np.abs(O.activation(z.numpy(), True)[0] - torch.nn.functional.gelu(z).numpy()).max() < 1e-14


# ------------------------------------------------------------------- refusals

_BUFFER = ctypes.create_string_buffer(64 + 16)


def _address():
    a = ctypes.addressof(_BUFFER)
    return a + (-a) % 16


def _status(fn, *args):
    try:
        fn(*args, kind="host")
    except R.RtccError as e:
        return e.status, str(e)
    return R.RTCC_OK, ""


def _norm(**kw):
    p = _address()
    d = R.rtcc_layer_norm_desc(abi_version=R.RTCC_ABI_VERSION, precision=R.RTCC_PREC_BF16, rows=5, channels=64, eps=1e-5, x=p,
                               out=p, x_stride=64, residual_stride=64, sum_out_stride=64, out_stride=64)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _norm_grad(fwd=None, **kw):
    p = _address()
    g = R.rtcc_layer_norm_grad_desc(fwd=_norm(**(fwd or {})), dout=p, dx=p, dout_stride=64, dsum_stride=64, dx_stride=64,
                                    dweight=p)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def _ffn(**kw):
    p = _address()
    d = R.rtcc_gated_ffn_desc(abi_version=R.RTCC_ABI_VERSION, precision=R.RTCC_PREC_BF16, rows=5, channels=64, hidden=128,
                              activation=R.RTCC_ACT_SILU, x=p, w_gate=p, w_up=p, w_down=p, out=p, x_stride=64, w_gate_stride=64,
                              w_up_stride=64, w_down_stride=128, out_stride=64, hidden_stride=128)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _ffn_grad(fwd=None, **kw):
    p = _address()
    g = R.rtcc_gated_ffn_grad_desc(fwd=_ffn(**dict(dict(gate=p, up=p, act=p), **(fwd or {}))), dout=p, dx=p, dw_gate=p, dw_up=p,
                                   dw_down=p, dout_stride=64, dx_stride=64, dw_gate_stride=64, dw_up_stride=64,
                                   dw_down_stride=128)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def test_good_descriptions_pass_the_checks():
    """All that is left is the missing GPU."""
    for call, d, rest in ((R.rtcc_layer_norm, _norm(), ()), (R.rtcc_layer_norm_grad, _norm_grad(), (0, 0)),
                          (R.rtcc_gated_ffn, _ffn(), (0, 0)), (R.rtcc_gated_ffn_grad, _ffn_grad(), (0, 0)),
                          (R.rtcc_layer_norm, _norm(channels=16384, x_stride=16384, out_stride=16384), ()),
                          (R.rtcc_gated_ffn, _ffn(rows=1, x_stride=-1, out_stride=0), (0, 0)),
                          (R.rtcc_gated_ffn_grad, _ffn_grad(dx=None, dw_gate=None, dw_up=None, dw_down=None), (0, 0)),
                          (R.rtcc_gated_ffn_grad, _ffn_grad(fwd=dict(out=None)), (0, 0))):
        assert _status(call, d, *rest)[0] == R.RTCC_E_STATE


def test_no_rows_are_no_work():
    none = dict(rows=0, x=None, out=None)
    assert _status(R.rtcc_layer_norm, _norm(**none))[0] == R.RTCC_OK
    assert _status(R.rtcc_gated_ffn, _ffn(w_gate=None, w_up=None, w_down=None, **none), 0, 0)[0] == R.RTCC_OK


@pytest.mark.parametrize("kw,name", [
    (dict(abi_version=5), "abi_version"), (dict(precision=2), "precision"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"),
    (dict(channels=0), "channels"), (dict(channels=12), "channels"), (dict(channels=16392), "channels"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(x=None), "x is NULL"), (dict(out=None), "out is NULL"),
    (dict(x=_address() + 2), "aligned"), (dict(x_stride=56), "stride"), (dict(out_stride=66), "alignment"),
    (dict(x_stride=(1 << 22) + 8), "stride"), (dict(residual=_address(), residual_stride=8), "residual"),
    (dict(sum_out=_address()), "one tensor"),
])
def test_layer_norm_refusals(kw, name):
    status, message = _status(R.rtcc_layer_norm, _norm(**kw))
    assert status == R.RTCC_E_ARG and name in message


@pytest.mark.parametrize("kw,name", [
    (dict(fwd=dict(x=None)), "x is NULL"), (dict(fwd=dict(residual=_address())), "sum_out is NULL"), (dict(dout=None), "dout"),
    (dict(dx=None), "dx"), (dict(dx_stride=32), "dx"), (dict(dsum=_address(), dsum_stride=68), "dsum"),
    (dict(fwd=dict(channels=4)), "channels"),
])
def test_layer_norm_gradient_refusals(kw, name):
    status, message = _status(R.rtcc_layer_norm_grad, _norm_grad(**kw), 0, 0)
    assert status == R.RTCC_E_ARG and name in message


@pytest.mark.parametrize("kw,name", [
    (dict(abi_version=7), "abi_version"), (dict(precision=-1), "precision"), (dict(rows=-1), "rows"),
    (dict(rows=(1 << 31) - 255), "rows"), (dict(rows=1 << 30, hidden=2048), "rows * width"),
    (dict(channels=20), "channels"), (dict(channels=65544), "channels"), (dict(hidden=4), "hidden"), (dict(hidden=0), "hidden"),
    (dict(activation=2), "activation"), (dict(gate=_address()), "all of them"), (dict(gate=_address(), act=_address()), "all of"),
    (dict(x=None), "x is NULL"), (dict(w_gate=None), "w_gate"), (dict(w_up=None), "w_up"), (dict(w_down=None), "w_down"),
    (dict(out=None), "out"), (dict(w_down_stride=64), "w_down"), (dict(w_gate_stride=100), "w_gate"),
    (dict(x=_address() + 8), "aligned"), (dict(out_stride=(1 << 22) + 8), "out"),
    (dict(gate=_address(), up=_address(), act=_address(), hidden_stride=64), "gate"),
])
def test_gated_ffn_refusals(kw, name):
    for call in (R.rtcc_gated_ffn, R.rtcc_gated_ffn_workspace):
        status, message = _status(call, _ffn(**kw), *((0, 0) if call is R.rtcc_gated_ffn else ()))
        assert status == R.RTCC_E_ARG and name in message


@pytest.mark.parametrize("kw,name", [
    (dict(fwd=dict(gate=None, up=None, act=None)), "gate, up and act"), (dict(fwd=dict(up=None)), "all of them"),
    (dict(dout=None), "dout"), (dict(dx_stride=8), "dx"), (dict(dw_gate_stride=0), "dw_gate"), (dict(dw_up_stride=65), "dw_up"),
    (dict(dw_down_stride=64), "dw_down"), (dict(fwd=dict(w_down=None)), "w_down"),
])
def test_gated_ffn_gradient_refusals(kw, name):
    status, message = _status(R.rtcc_gated_ffn_grad, _ffn_grad(**kw), 0, 0)
    assert status == R.RTCC_E_ARG and name in message


class On:
    """A tensor that says it is on a GPU."""

    def __init__(self, x, device=0):
        self.x, self.device = x, device

    def get_device(self):
        return self.device

    def __getattr__(self, name):
        return getattr(self.x, name)


def _tensors():
    x, h, w = torch.zeros(4, 16), torch.zeros(4, 24), torch.zeros(24, 16)
    norm = dict(x=x, out=x, weight=x[0], bias=x[0], residual=x, sum_out=torch.zeros(4, 16))
    unit = dict(x=x, w_gate=w, w_up=w, w_down=torch.zeros(16, 24), out=x, gate=h, up=h, act=h)
    return norm, unit


@pytest.mark.parametrize("which,make", [(0, R.layer_norm_desc), (1, R.gated_ffn_desc)])
def test_tensors_of_two_devices(which, make):
    t = _tensors()[which]
    d = make(**{k: On(v) for k, v in t.items()})
    for name in t:
        with pytest.raises(ValueError, match="another device"):
            make(**{k: v if k == name else On(v) for k, v in t.items()})
    for grad, names in ((R.layer_norm_grad_desc, ("dout", "dx", "dsum")), (R.gated_ffn_grad_desc, ("dout", "dx"))):
        if (grad is R.layer_norm_grad_desc) == (which == 0):
            grad(d, **{n: On(t["x"]) for n in names})
            for name in names:
                with pytest.raises(ValueError, match="another device"):
                    grad(d, **{n: t["x"] if n == name else On(t["x"]) for n in names})


def test_another_device_than_the_current_one_is_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    norm, unit = ({k: On(v, 1) for k, v in t.items()} for t in _tensors())
    n, u, x = R.layer_norm_desc(**norm), R.gated_ffn_desc(**unit), norm["x"]
    for call, d, rest in ((R.rtcc_layer_norm, n, ()), (R.rtcc_layer_norm_grad, R.layer_norm_grad_desc(n, x, x), (0, 0)),
                          (R.rtcc_gated_ffn, u, (0, 0)), (R.rtcc_gated_ffn_grad, R.gated_ffn_grad_desc(u, x, x), (0, 0))):
        with pytest.raises(ValueError, match="current device"):
            call(d, *rest)


def test_host_tensors_reach_the_host_library_only():
    norm, unit = _tensors()
    n, u, x = R.layer_norm_desc(**norm), R.gated_ffn_desc(**unit), norm["x"]
    for call, d, rest in ((R.rtcc_layer_norm, n, ()), (R.rtcc_layer_norm_grad, R.layer_norm_grad_desc(n, x, x), (0, 0)),
                          (R.rtcc_gated_ffn, u, (0, 0)), (R.rtcc_gated_ffn_grad, R.gated_ffn_grad_desc(u, x, x), (0, 0))):
        with pytest.raises(ValueError, match="host memory"):
            call(d, *rest)
        with pytest.raises(R.RtccError) as e:
            call(d, *rest, kind="host")
        assert e.value.status == R.RTCC_E_STATE or "aligned" in str(e.value)


def test_wrong_shapes_and_types():
    norm, unit = _tensors()
    n, u = R.layer_norm_desc(**norm), R.gated_ffn_desc(**unit)
    x = norm["x"]
    for kw in (dict(x=x[0]), dict(out=torch.zeros(5, 16)), dict(out=x.bfloat16()), dict(x=x.t()), dict(weight=torch.zeros(15)),
               dict(bias=torch.zeros(16).bfloat16()), dict(x=x.double())):
        with pytest.raises(ValueError):
            R.layer_norm_desc(**dict(norm, **kw))
    for kw in (dict(x=x[0]), dict(w_up=torch.zeros(16, 16)), dict(w_down=torch.zeros(24, 16)), dict(out=torch.zeros(4, 24)),
               dict(w_gate=torch.zeros(16, 24).t()), dict(act=torch.zeros(4, 48)[:, :24]), dict(gate=torch.zeros(4, 16))):
        with pytest.raises(ValueError):
            R.gated_ffn_desc(**dict(unit, **kw))
    for make, fwd in ((R.layer_norm_grad_desc, n), (R.gated_ffn_grad_desc, u)):
        for dout, dx in ((x.bfloat16(), x), (x, x[:3]), (x, x.bfloat16())):
            with pytest.raises(ValueError):
                make(fwd, dout, dx)
