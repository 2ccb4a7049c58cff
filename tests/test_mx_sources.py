"""The microscaled kernels' sources: no access that promises the compiler more alignment than its address has."""
import glob
import os
import subprocess

import pytest

from paper_1805_07941_amd import build

SOURCES = sorted(glob.glob(os.path.join(build.CSRC, "mx_*.hip")))


@pytest.mark.parametrize("source", SOURCES, ids=os.path.basename)
def test_no_alignment_is_lost_on_the_way(source):
    """Rows of values lie at any address of their type; a pointer that drops this from its type lets the compiler count on 16 bytes."""
    r = subprocess.run([build._hipcc()] + build.FLAGS + ["-Werror=align-mismatch", "--cuda-device-only", "-fsyntax-only", source],
                       capture_output=True, text=True)
    assert r.returncode == 0, "\n".join(l for l in r.stderr.splitlines() if "error" in l)


def test_there_are_sources():
    assert len(SOURCES) >= 4
