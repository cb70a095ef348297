"""torch may bring a HIP runtime of its own: whichever of torch and the binding is imported first, the process has one runtime,
and both work on it.  (With two, the second one finds no device, and what the first made is unknown to it.)"""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ORDERS = ["from paper_2607_22614_amd import dr\nimport torch", "import torch\nfrom paper_2607_22614_amd import dr"]


def _child(code):
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=110, cwd=ROOT)
    assert r.returncode == 0, r.stderr
    return r.stdout


@pytest.mark.parametrize("imports", ORDERS)
def test_one_runtime_is_loaded(imports):
    out = _child(imports + """
paths = {line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line or "libhsa-runtime64" in line}
print(sorted(paths))
""")
    assert out.count("libamdhip64") == 1 and out.count("libhsa-runtime64") == 1, out


@pytest.mark.gpu
@pytest.mark.parametrize("imports", ORDERS)
def test_both_use_the_gpu(imports):
    print("[gpu] imports", imports.splitlines(), flush=True)
    _child(imports + """
x = torch.full((3, 200), 3.0, device="cuda")
q = dr.QMatrix.empty(3, 200)
dr.dr_quantize(x, q)
assert (q.data[:, :200].view(torch.float8_e4m3fn).float() == 384.0).all() and (q.scales[0, :, :2] == 120).all()
""")
