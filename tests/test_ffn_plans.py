"""Tiles that the feed-forward unit's products take (the host's choice, without a
GPU), at the sizes where tests on the GPU count on them."""

import os
import subprocess

import pytest

from paper_2608_08330_amd import build as B
from tests.test_gpu_ffn_large import CASES, STRIDES

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")
UNITS = 256


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plans") / "ffn_plans")
    subprocess.run([B.CXX] + B.HOST_FLAGS + [os.path.join(NATIVE, "ffn_plans.cpp"), "-o", exe], check=True)
    return exe


@pytest.fixture
def plans(program):
    def ask(rows, channels, hidden, strides=None, bf16=True):
        """product: (tile, slices, blocks)."""
        strides = strides or (channels, channels)
        out = subprocess.run([program] + [str(int(v)) for v in (bf16, rows, channels, hidden, *strides)], check=True,
                             stdout=subprocess.PIPE, text=True).stdout
        return {line.split()[0]: tuple(int(v) for v in line.split()[1:]) for line in out.splitlines()}

    return ask


@pytest.mark.parametrize("size,products,train", CASES)
def test_largest_tiles_one_after_another(plans, size, products, train):
    p = plans(*size)
    for product in products:
        tile, slices, blocks = p[product.replace("_sliced", "")]
        assert tile == 256 and blocks > UNITS and (slices > 1) == product.endswith("_sliced")
        assert train or product in ("gated", "down", "down_sliced")


def test_every_form_of_the_product_is_there():
    """Stores of a tile's end: h; h, g and u; plain; slices; dG and dU.  Operands: rows,
    rows; rows, columns, in two segments; columns, columns."""
    assert {p for _, products, _ in CASES for p in products} == {
        "gated", "gated_saved", "down", "down_sliced", "dhidden", "dx", "dx_sliced", "weights", "weights_sliced"}


def test_strides_decide_the_tiles_of_dx(plans):
    rows, channels, hidden = STRIDES
    one, two = (plans(rows, channels, hidden, s) for s in ((channels + 16, channels + 16), (channels + 16, channels + 48)))
    assert one["dx"][0] == 256 and two["dx"][0] < 256
    # what no tile of two strides may ever be
    for size in ((12400, 2056, 2056), (22801, 136, 3512), (121275, 136, 8), (16384, 2048, 8192)):
        p = plans(*size, (size[1] + 16, size[1] + 48))
        assert p.get("dx", p.get("dx_shared"))[0] < 256


def test_most_tiles(program):
    """Half tiles of 64 x 32 of a gated product, 2^40 / 520 rows of 520: more than 2^29."""
    most = int(subprocess.run([program], check=True, stdout=subprocess.PIPE, text=True).stdout)
    assert most == -(-(2 ** 40 // 520) // 64) * 17 == 561649570 < 1 << 30
