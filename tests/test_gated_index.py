"""What the products of a gated block copy to LDS of the fused weights, on the CPU.

Walks every tile with the kernel's own functions (csrc/product_index.h): a stage's rows are the right rows of gate and up, those
behind gate's last one are outside of their buffer, not the beginning of up, and scale codes are those of their rows also where
up's first row lies inside a square block.
"""
import pytest

from tests.native_build import MISSING, native, run

pytestmark = pytest.mark.skipif(MISSING, reason="g++ or the HIP headers not available")


@pytest.fixture(scope="module")
def gated_check(tmp_path_factory):
    return native(str(tmp_path_factory.mktemp("gated") / "gated_check"), "gated_check.cpp")


@pytest.mark.parametrize("tile", [128, 256])
@pytest.mark.parametrize("sh", [0, 7])
@pytest.mark.parametrize("f,cols", [(1, 100), (64, 600), (130, 512), (128, 1025), (345, 300), (513, 129)])
def test_copies_are_of_their_pairs(gated_check, f, cols, sh, tile):
    run(gated_check, f, cols, sh, tile)
