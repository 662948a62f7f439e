"""The operators' sources and launches, looked at on the host (no GPU)."""
import os
import subprocess

import pytest

from paper_2609_03311_amd import _build


@pytest.mark.parametrize("source", ["rows.hip", "qproduct.hip", "rotary.hip"])
def test_pointers_keep_their_alignment(source):
    """Rows start at any element, so no load or store may be taken to lie on
    its own size: a place handed on as a type of larger alignment is a
    warning of the compiler's, which the build takes for an error."""
    assert "-Werror=align-mismatch" in _build.FLAGS
    r = subprocess.run(
        [_build.hipcc(), *_build.FLAGS, "-fsyntax-only",
         os.path.join(_build.CSRC, source)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
