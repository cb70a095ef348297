"""Quantization's streamed loads are loads of whole, aligned 16 bytes: the sources that are streamed have rows made of such
pieces, the last one included (csrc/quant_kernels.h, as the launch calls it)."""
import pytest

from tests.native_build import MISSING, native, run

pytestmark = pytest.mark.skipif(MISSING, reason="g++ or the HIP headers not available")


def test_streamed_loads_are_aligned(tmp_path):
    run(native(str(tmp_path / "quantize_check"), "quantize_check.cpp"))
