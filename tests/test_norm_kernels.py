"""The layer norm kernels of the built library: one for every way in which a row of
some width is cut, and no other."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2608_08330_amd import build as B

NM = shutil.which("nm") or "/opt/rocm/llvm/bin/llvm-nm"


def _cut(channels, most):
    """Threads and eights of channels each: the fewest threads that hold the row."""
    eights = channels // 8
    g = next((g for g in (8, 16, 32, 64, 256, 512) if eights <= most * g), 512)
    return g, -(-eights // g)


def _cuts(most):
    return {_cut(c, most) for c in range(8, 16384 + 1, 8)}


@pytest.mark.skipif(not os.path.exists(NM), reason="no symbol lister")
def test_kernels_that_rows_take():
    library = os.path.join(B.LIB, "librtcc.so")
    if not os.path.exists(library):
        B.build()
    names = subprocess.run([NM, "-C", library], check=True, stdout=subprocess.PIPE, text=True).stdout
    forward = set(re.findall(r"__device_stub__k_layer_norm<([\w ]+), (\d+), (\d+)>", names))
    backward = set(re.findall(r"__device_stub__k_layer_norm_grad<([\w ]+), (\d+), (\d+), (\w+)>", names))
    types = ("unsigned short", "float")
    assert forward == {(t, str(g), str(v)) for t in types for g, v in _cuts(4)}
    # three eights at most, of float32 with a gradient past the norm two
    assert backward == {(t, str(g), str(v), past) for t in types for past in ("true", "false")
                        for g, v in _cuts(2 if (t, past) == ("float", "true") else 3)}
