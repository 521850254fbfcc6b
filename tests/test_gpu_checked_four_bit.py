"""The bounds-checked flavour (tests/test_gpu_checked.py) on 4-bit caches and windows: no check fires, which bkv_sync
would report, and the results match the 64-bit references."""
import subprocess
import sys

import pytest

from tests.test_gpu_checked import ROOT, _checked_env

pytestmark = pytest.mark.gpu


def test_checked_flavour_four_bit_and_window_run_clean():
    tests = ["tests/test_gpu_four_bit.py", "tests/test_gpu_four_bit_range.py", "tests/test_gpu_window.py",
             "tests/test_gpu_evict_select.py"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", *tests], cwd=ROOT,
                       env=_checked_env(), capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
