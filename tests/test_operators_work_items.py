"""What the attention makes of the records of its work list, on the host (plain g++ with AddressSanitizer + UBSan, no GPU code)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_records_lead_nowhere_outside_whatever_they_hold(tmp_path):
    exe, csrc = str(tmp_path / "items"), os.path.join(ROOT, "paper_2504_02921_amd", "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                        os.path.join(ROOT, "tests", "operators_items_driver.cpp"), os.path.join(csrc, "hr_pair_host.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)          # the sanitizer runtime must come first in the link order
    r = subprocess.run([exe], capture_output=True, text=True, env=env)
    assert r.returncode == 0 and "inside" in r.stdout, (r.stdout + r.stderr)[-2000:]
