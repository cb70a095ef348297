"""What the tiled products copy to LDS, block by block, on the CPU.

Walks a workgroup's items with the kernel's own functions (csrc/product_index.h): every copy of an item reads the block it should,
rows past a matrix are outside of their buffer, and no copy, those for tiles outside of c and those behind the
last item among them, has a scalar offset beyond its buffer's length or reads outside of its matrix.
"""
import pytest

from tests.native_build import MISSING, native, run

pytestmark = pytest.mark.skipif(MISSING, reason="g++ or the HIP headers not available")


@pytest.fixture(scope="module")
def product_check(tmp_path_factory):
    return native(str(tmp_path_factory.mktemp("product") / "product_check"), "product_check.cpp")


@pytest.mark.parametrize("tile,quarters", [(128, 0), (128, 1), (256, 0)])
@pytest.mark.parametrize("ahead", [2, 4])
@pytest.mark.parametrize("rows_a,rows_b,cols", [(1, 1, 600), (128, 129, 512), (257, 300, 1000), (300, 640, 1025), (513, 127, 520)])
@pytest.mark.parametrize("sh_a,sh_b", [(0, 7), (0, 0), (7, 7)])
def test_copies_stay_in_their_matrices(product_check, rows_a, rows_b, cols, sh_a, sh_b, tile, quarters, ahead):
    run(product_check, rows_a, rows_b, cols, sh_a, sh_b, tile, quarters, ahead)
