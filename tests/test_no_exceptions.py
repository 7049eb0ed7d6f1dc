"""What every launch passes through on its way from a C entry neither allocates nor throws: an exception there would end the caller's process."""
import os
import shutil
import subprocess

import pytest

from paper_2604_06483_amd import build

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None or shutil.which("nm") is None, reason="needs hipcc and nm")


def test_the_launches_shared_setup_cannot_throw(tmp_path):
    out = tmp_path / "ll_api.o"
    subprocess.run(["hipcc", *build.FLAGS, "-c", os.path.join(build.HERE, "csrc", "ll_api.hip"), "-o", str(out)], check=True, capture_output=True)
    wanted = subprocess.run(["nm", "-u", str(out)], check=True, capture_output=True, text=True).stdout.split()
    assert not [n for n in wanted if n.startswith(("_Znw", "_Zna", "__cxa_throw", "_ZSt20__throw", "_ZSt17__throw"))], wanted
