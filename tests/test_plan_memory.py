"""Plans whose device memory cannot be had, on the CPU: every allocation and every copy of a plan's creation fails in turn
(tests/native/plan_memory_check.cpp)."""
import pytest

from tests.native_build import MISSING, native, run

pytestmark = pytest.mark.skipif(MISSING, reason="g++ or the HIP headers not available")
SOURCES = ("plan.cpp", "capi.cpp", "staging.cpp", "reshard.cpp", "relay.cpp", "moments.cpp")


def test_memory_is_taken_before_anything_is_copied(tmp_path):
    run(native(str(tmp_path / "plan_memory_check"), "plan_memory_check.cpp", SOURCES))
