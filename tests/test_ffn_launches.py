"""Launch sizes of the feed-forward unit at the limits of its description (the
host's arithmetic, without a GPU), and the refusal past them."""

import os
import subprocess

from paper_2608_08330_amd import build as B
from paper_2608_08330_amd import rtcc as R
from tests.test_oracle_blocks import _ffn, _status

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")


def test_launches_at_the_limits(tmp_path):
    exe = str(tmp_path / "ffn_launches")
    subprocess.run([B.CXX] + B.HOST_FLAGS + [os.path.join(NATIVE, "ffn_launches.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stdout


def test_most_rows_and_values():
    most = (1 << 31) - 256
    for rows, hidden, status in ((most, 128, R.RTCC_E_STATE), (most + 1, 128, R.RTCC_E_ARG), ((1 << 40) // 1024, 1024, R.RTCC_E_STATE),
                                 ((1 << 40) // 1024 + 1, 1024, R.RTCC_E_ARG)):
        d = _ffn(rows=rows, hidden=hidden, w_down_stride=hidden, hidden_stride=hidden)
        assert _status(R.rtcc_gated_ffn, d, 0, 0)[0] == status
