"""The token operators' oracle against differences and against library
routines, and the operators' refusals (host test library: the checks are the
GPU library's, the launchers only report that there is no GPU)."""

import ctypes

import numpy as np
import pytest

from oracle import tokens as T
from paper_2608_08330_amd import rtcc as R


# --------------------------------------------------------------------- oracle

@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_complex_numbers(interleaved):
    rng = np.random.default_rng(0)
    x = rng.normal(size=(5, 3, 16))
    ang = rng.uniform(-9, 9, (5, 8))
    i, j = T._pairs(16, interleaved)
    z = (x[..., i] + 1j * x[..., j]) * np.exp(1j * ang)[:, None]
    y = T.rotate(x, ang, interleaved)
    assert np.abs(y[..., i] - z.real).max() < 1e-14 and np.abs(y[..., j] - z.imag).max() < 1e-14
    assert np.abs(T.rotate(y, -ang, interleaved) - x).max() < 1e-14


def test_norm_rope_gradient_against_differences():
    rng = np.random.default_rng(1)
    x, w, dy = rng.normal(size=(4, 2, 16)), rng.normal(size=16), rng.normal(size=(4, 2, 16))
    ang = rng.uniform(-3, 3, (4, 8))
    dx, dw = T.norm_rope_grad(x, w, ang, 1e-3, False, dy)

    def loss(x, w):
        return (T.norm_rope(x, w, ang, 1e-3, False) * dy).sum()

    h = 1e-5  # central differences: error of order h^2 = 1e-10
    for at in np.ndindex(*x.shape):
        step = np.zeros_like(x)
        step[at] = h
        assert abs((loss(x + step, w) - loss(x - step, w)) / (2 * h) - dx[at]) < 1e-8
    for d in range(16):
        step = np.zeros(16)
        step[d] = h
        assert abs((loss(x, w + step) - loss(x, w - step)) / (2 * h) - dw.sum(0)[d]) < 1e-8


_SEQS = [(0, 3, 0, 5, 2), (3, 2, 5, 1, 0), (5, 0, 6, 2, 1), (5, 4, 8, 4, 0)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("softcap,bias", [(0.0, False), (1.5, True)])
def test_attention_gradient_against_differences(causal, softcap, bias):
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(9, 4, 8)), rng.normal(size=(12, 2, 8)), rng.normal(size=(12, 2, 8))
    do = rng.normal(size=q.shape)
    kw = dict(causal=causal, slopes=rng.uniform(0, 1, 4) if bias else None, scale=0.7, softcap=softcap)

    def loss(q, k, v):
        return np.nansum(T.Attention(q, k, v, _SEQS, **kw).out * do)

    grads, _ = T.Attention(q, k, v, _SEQS, **kw).grad(do)
    h = 1e-5
    for which, grad in enumerate(grads):
        args = [q, k, v]
        for at in list(np.ndindex(*args[which].shape))[::3]:
            lo, hi = [x.copy() for x in args], [x.copy() for x in args]
            lo[which][at] -= h
            hi[which][at] += h
            assert abs((loss(*hi) - loss(*lo)) / (2 * h) - grad[at]) < 1e-8


def test_attention_oracle_against_torch():
    import torch
    rng = np.random.default_rng(3)
    q, k, v = (rng.normal(size=(6, 2, 8)) for _ in range(3))
    o = T.Attention(q, k, v, [(0, 6, 0, 6, 0)], causal=True, scale=0.5)
    tq, tk, tv = (torch.from_numpy(x).permute(1, 0, 2) for x in (q, k, v))
    ref = torch.nn.functional.scaled_dot_product_attention(tq, tk, tv, is_causal=True, scale=0.5)
    assert np.abs(o.out - ref.permute(1, 0, 2).numpy()).max() < 1e-14


def test_rows_without_keys_and_limits():
    assert T.limits(4, 2, True, 0) == [0, 0, 1, 2]
    assert T.limits(3, 5, True, 4) == [4, 4, 5]
    assert T.limits(2, 3, False, 0) == [3, 3]
    o = T.Attention(np.ones((4, 1, 8)), np.ones((2, 1, 8)), np.ones((2, 1, 8)), [(0, 4, 0, 2, 0)], causal=True)
    assert (o.out[:2] == 0).all() and (o.lse[0, :2] == -np.inf).all() and np.isfinite(o.lse[0, 2:]).all()


# ------------------------------------------------------------------- refusals

_MEM = np.zeros(1 << 14, np.float64)  # 16-byte aligned below; never touched by the host library


def _address():
    return (_MEM.ctypes.data + 15) // 16 * 16


def _rope(**kw):
    p = _address()
    d = R.rtcc_norm_rope_desc(abi_version=R.RTCC_ABI_VERSION, precision=R.RTCC_PREC_BF16, rows=3, q_heads=2,
                              kv_heads=1, head_dim=32, n_axes=2, eps=1e-6, q=p, k=p, q_out=p, k_out=p, positions=p,
                              inv_freq=p)
    d.sections[:] = (6, 10, 0)
    for name in ("q_stride", "k_stride", "v_stride", "q_out_stride", "k_out_stride", "v_out_stride"):
        getattr(d, name)[:] = (64, 32)
    for name, value in kw.items():
        if isinstance(value, tuple):
            getattr(d, name)[:] = value
        else:
            setattr(d, name, value)
    return d


def _attn(**kw):
    p = _address()
    d = R.rtcc_attn_desc(abi_version=R.RTCC_ABI_VERSION, precision=R.RTCC_PREC_FP32, n_seqs=1, q_heads=4, kv_heads=2,
                         head_dim=64, scale=0.125, q_rows=5, k_rows=7, q_offsets=p, k_offsets=p, k_lens=p, q=p, k=p,
                         v=p, out=p, lse=p)
    for name in ("q_stride", "out_stride"):
        getattr(d, name)[:] = (256, 64)
    for name in ("k_stride", "v_stride"):
        getattr(d, name)[:] = (128, 64)
    for name, value in kw.items():
        if isinstance(value, tuple):
            getattr(d, name)[:] = value
        else:
            setattr(d, name, value)
    return d


def _status(call, *args):
    try:
        call(*args, kind="host")
    except R.RtccError as e:
        return e.status, str(e)
    return 0, ""


_NAN, _INF = float("nan"), float("inf")


def test_valid_descriptions_reach_the_launcher():
    assert _status(R.rtcc_norm_rope, _rope())[0] == R.RTCC_E_STATE
    assert _status(R.rtcc_attention, _attn(), 0, 0)[0] == R.RTCC_E_STATE
    # nothing to do: no launch, and nothing is looked at
    assert _status(R.rtcc_norm_rope, _rope(rows=0, q=None, k=None, q_out=None, k_out=None))[0] == 0
    assert _status(R.rtcc_attention, _attn(n_seqs=0, q=None, q_offsets=None), 0, 0)[0] == 0
    assert _status(R.rtcc_attention, _attn(q_rows=0, q=None, out=None), 0, 0)[0] == 0
    # one head, one row: their strides are not looked at
    assert _status(R.rtcc_norm_rope, _rope(rows=1, kv_heads=1, k_stride=(-1, 3), k_out_stride=(0, 0)))[0] == R.RTCC_E_STATE
    # no keys at all
    assert _status(R.rtcc_attention, _attn(k_rows=0, k=None, v=None), 0, 0)[0] == R.RTCC_E_STATE
    # only keys to norm
    assert _status(R.rtcc_norm_rope, _rope(q_heads=0, q=None, q_out=None))[0] == R.RTCC_E_STATE


@pytest.mark.parametrize("bad,word", [
    (dict(abi_version=1), "abi_version"), (dict(precision=7), "precision"), (dict(head_dim=24), "head_dim"),
    (dict(head_dim=144), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(rows=-1), "rows"),
    (dict(rows=1 << 31), "rows"), (dict(q_heads=-1), "heads"), (dict(q_heads=0, kv_heads=0), "heads"),
    (dict(kv_heads=1025), "heads"), (dict(interleaved=2), "interleaved"), (dict(n_axes=0), "n_axes"),
    (dict(n_axes=4), "n_axes"), (dict(sections=(8, 9, 0)), "pairs"), (dict(sections=(-1, 9, 0)), "section"),
    (dict(sections=(2147483647, 2147483647, 0)), "section"), (dict(eps=-1.0), "eps"), (dict(eps=_NAN), "eps"),
    (dict(eps=_INF), "eps"), (dict(q=None), "q is NULL"), (dict(k=None), "k is NULL"),
    (dict(q_out=None), "q_out is NULL"), (dict(k_out=None), "k_out is NULL"), (dict(positions=None), "positions"),
    (dict(inv_freq=None), "inv_freq"), (dict(q_stride=(0, 32)), "stride"), (dict(q_stride=(64, 16)), "stride"),
    (dict(q_stride=(68, 32)), "alignment"), (dict(q_out_stride=(1 << 23, 32)), "stride"),
    (dict(q_stride=(-64, 32)), "stride"), (dict(q_weight_per_head=2), "weight"), (dict(v=16, v_out=16), "v without slots"),
    (dict(slots=16, slot_rows=-1), "slot_rows"), (dict(slots=16, slot_rows=4, v=16), "v_out is NULL"),
])
def test_norm_rope_refusals(bad, word):
    status, message = _status(R.rtcc_norm_rope, _rope(**bad))
    assert status == R.RTCC_E_ARG and word in message


def test_norm_rope_misaligned_pointer():
    status, message = _status(R.rtcc_norm_rope, _rope(q=_address() + 8))
    assert status == R.RTCC_E_ARG and "aligned" in message


@pytest.mark.parametrize("bad,word", [
    (dict(abi_version=0), "abi_version"), (dict(precision=-1), "precision"), (dict(head_dim=40), "head_dim"),
    (dict(n_seqs=-1), "n_seqs"), (dict(n_seqs=65537), "n_seqs"), (dict(q_heads=3), "multiple"),
    (dict(kv_heads=0), "heads"), (dict(q_heads=0), "heads"), (dict(q_heads=2048), "heads"), (dict(causal=2), "causal"),
    (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=_NAN), "scale"), (dict(scale=_INF), "scale"),
    (dict(softcap=-1.0), "softcap"), (dict(softcap=_NAN), "softcap"), (dict(softcap=_INF), "softcap"),
    (dict(q_rows=-1), "q_rows"), (dict(q_rows=1 << 30), "q_rows"), (dict(k_rows=-1), "k_rows"),
    (dict(k_rows=1 << 31), "k_rows"), (dict(prefix_lens=16), "prefix"), (dict(q=None), "q is NULL"),
    (dict(k=None), "k is NULL"), (dict(v=None), "v is NULL"), (dict(out=None), "out is NULL"),
    (dict(q_offsets=None), "q_offsets"), (dict(k_offsets=None), "k_offsets"), (dict(k_stride=(0, 64)), "stride"),
    (dict(v_stride=(128, 65)), "alignment"), (dict(out_stride=(256, 32)), "stride"),
    (dict(k_stride=((1 << 22) + 64, 64)), "stride"),
])
def test_attention_refusals(bad, word):
    status, message = _status(R.rtcc_attention, _attn(**bad), 0, 0)
    assert status == R.RTCC_E_ARG and word in message
    # the workspace question is refused in the same way
    with pytest.raises(R.RtccError):
        R.rtcc_attention_workspace(_attn(**bad), kind="host")


def test_gradient_refusals():
    p = _address()
    g = R.rtcc_attn_grad_desc(fwd=_attn(), dout=p, dq=p, dk=p, dv=p)
    for name in ("dout_stride", "dq_stride"):
        getattr(g, name)[:] = (256, 64)
    for name in ("dk_stride", "dv_stride"):
        getattr(g, name)[:] = (128, 64)
    assert _status(R.rtcc_attention_grad, g, 0, 0)[0] == R.RTCC_E_STATE
    for name in ("dout", "dq", "dk", "dv"):
        setattr(g, name, None)
        status, message = _status(R.rtcc_attention_grad, g, 0, 0)
        assert status == R.RTCC_E_ARG and name in message
        setattr(g, name, p)
    g.fwd.lse = None
    assert "lse" in _status(R.rtcc_attention_grad, g, 0, 0)[1]

    n = R.rtcc_norm_rope_grad_desc(fwd=_rope(), dq_out=p, dk_out=p, dq=p, dk=p)
    for name in ("dq_out_stride", "dk_out_stride", "dq_stride", "dk_stride"):
        getattr(n, name)[:] = (64, 32)
    assert _status(R.rtcc_norm_rope_grad, n, 0, 0)[0] == R.RTCC_E_STATE
    for name in ("dq_out", "dk_out", "dq", "dk"):
        setattr(n, name, p + 4)
        status, message = _status(R.rtcc_norm_rope_grad, n, 0, 0)
        assert status == R.RTCC_E_ARG and name in message
        setattr(n, name, p)


def test_null_descriptions():
    lib = R.load("host")
    n = ctypes.c_size_t()
    assert lib.rtcc_norm_rope(None, None) == R.RTCC_E_ARG
    assert lib.rtcc_norm_rope_grad(None, None, 0, None) == R.RTCC_E_ARG
    assert lib.rtcc_attention(None, None, 0, None) == R.RTCC_E_ARG
    assert lib.rtcc_attention_grad(None, None, 0, None) == R.RTCC_E_ARG
    assert lib.rtcc_norm_rope_grad_workspace(None, ctypes.byref(n)) == R.RTCC_E_ARG
    assert lib.rtcc_attention_workspace(None, ctypes.byref(n)) == R.RTCC_E_ARG
    assert lib.rtcc_attention_grad_workspace(None, ctypes.byref(n)) == R.RTCC_E_ARG
    d = _attn()
    assert lib.rtcc_attention_workspace(ctypes.byref(d), None) == R.RTCC_E_ARG


def test_binding_refuses_wrong_tensors():
    import torch
    q, k = torch.zeros(4, 2, 32), torch.zeros(4, 1, 32)
    off = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        R.attention_desc(q.half(), k, k, q, off, off)
    with pytest.raises(ValueError):
        R.attention_desc(q, k.bfloat16(), k, q, off, off)
    with pytest.raises(ValueError):
        R.attention_desc(q, k, k[:3], q, off, off)
    with pytest.raises(ValueError):
        R.attention_desc(q, k, k, q, off.long(), off)
    with pytest.raises(ValueError):
        R.attention_desc(q, k, k, q, off, off, slopes=torch.zeros(3))
    with pytest.raises(ValueError):
        R.attention_desc(q.transpose(1, 2).contiguous().transpose(1, 2), k, k, q, off, off)
    pos, f = torch.zeros(4, 1), torch.zeros(16)
    with pytest.raises(ValueError):
        R.norm_rope_desc(q, k, q, k, None, None, pos, torch.zeros(15), (16,))
    with pytest.raises(ValueError):
        R.norm_rope_desc(q, k, q, k, torch.zeros(31), None, pos, f, (16,))
    with pytest.raises(ValueError):
        R.norm_rope_desc(None, None, None, None, None, None, pos, f, (16,))
    with pytest.raises(ValueError):
        R.norm_rope_desc(q, k, q, k[:3], None, None, pos, f, (16,))
