"""The binding imports wherever torch does (not gpu)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_import_needs_no_device_support_of_torch():
    """A torch that was built without a GPU has none of the device functions."""
    code = ("import torch\n"
            "for n in [n for n in dir(torch._C) if n.startswith('_cuda_') and n != '_cuda_isDriverSufficient']:\n"
            "    delattr(torch._C, n)\n"
            "import paper_2603_19610_amd as pv\n"
            "assert pv.lib().pvlm_version() == 1\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
