"""Every kernel source passes the compiler's front end for gfx950 without a warning, under the flags of the
build. CPU only (nothing is generated)."""
import glob
import os
import shutil
import subprocess

import pytest

from paper_2505_07531_amd import _build

SOURCES = sorted(os.path.basename(p) for p in glob.glob(os.path.join(_build.CSRC, "*.hip")))


@pytest.mark.parametrize("src", SOURCES)
def test_no_warnings(src):
    if shutil.which(_build.HIPCC) is None:
        pytest.skip("hipcc not available")
    r = subprocess.run([_build.HIPCC, *_build.COMMON, "-Werror", "-Wno-unused-command-line-argument", "-x", "hip",
                        "--cuda-device-only", "-fsyntax-only", os.path.join(_build.CSRC, src)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
