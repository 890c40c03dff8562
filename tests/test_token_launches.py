"""Launch sizes of the token operators at the limits of their descriptions (the
host's arithmetic, without a GPU), and the refusal past them."""

import os
import subprocess

from paper_2608_08330_amd import build as B
from paper_2608_08330_amd import rtcc as R
from tests.test_oracle_tokens import _address, _attn, _status

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")


def test_launches_at_the_limits(tmp_path):
    exe = str(tmp_path / "token_launches")
    subprocess.run([B.CXX] + B.HOST_FLAGS + [os.path.join(NATIVE, "token_launches.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stdout


def test_places_past_the_last_row_fit_an_int():
    """A tile's rows are counted up to 127 past the last one."""
    most = (1 << 31) - 256
    for name in ("q_rows", "k_rows"):
        for rows, status in ((most, R.RTCC_E_STATE), (most + 1, R.RTCC_E_ARG), ((1 << 31) - 1, R.RTCC_E_ARG)):
            got, message = _status(R.rtcc_attention, _attn(q_heads=1, kv_heads=1, **{name: rows}), 0, 0)
            assert got == status and (got != R.RTCC_E_ARG or name in message)


def test_more_keys_than_the_gradient_counts_are_refused():
    p = _address()
    for kv_heads, rows, status in ((1024, (1 << 25) - 1, R.RTCC_E_STATE), (1024, 1 << 25, R.RTCC_E_ARG)):
        g = R.rtcc_attn_grad_desc(fwd=_attn(q_heads=1024, kv_heads=kv_heads, head_dim=16, k_rows=rows), dout=p, dq=p, dk=p,
                                  dv=p)
        for d, names in ((g, ("dout_stride", "dq_stride", "dk_stride", "dv_stride")),
                         (g.fwd, ("q_stride", "k_stride", "v_stride", "out_stride"))):
            for name in names:
                getattr(d, name)[:] = (16 * 1024, 16)
        got, message = _status(R.rtcc_attention_grad, g, 0, 0)
        assert got == status and (got != R.RTCC_E_ARG or "kv_heads" in message)
