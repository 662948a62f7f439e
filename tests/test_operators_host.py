"""The operators' sources and launches, looked at on the host (no GPU)."""
import os
import subprocess

import pytest

from operator_launches import launches
from paper_2609_03311_amd import _build


def product(rows, cols, depth, dtype=0, **more):
    """A call with rows on 16-byte addresses, or as `more` says."""
    pitch = -(-depth // 16) * 16
    return ["dopr_quant_matmul", "_QuantMatmulArgs",
            dict(dtype=dtype, rows=rows, cols=cols, depth=depth, x=256,
                 x_row_stride=pitch, x_scale=256, w=256, w_row_stride=pitch,
                 w_scale=256, y=256, y_row_stride=cols) | more]


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


def test_dynamic_lds_is_asked_for_on_every_device():
    """The limit belongs to a device: each is asked once, and one that
    refused is asked again."""
    call = product(12900, 24576, 4096)
    got = launches([call + [dict(device=d, refuse=r)] for d, r in (
        (0, False), (0, False), (1, True), (1, False), (1, False),
        (0, False), (70, False), (70, False))])
    lds = got[0]["launches"][0]["lds"]
    assert lds > 64 * 1024
    asked = [[(d, size) for d, size, _ in g["limits"]] for g in got]
    assert asked == [[(0, lds)], [], [(1, lds)], [(1, lds)], [], [],
                     [(70, lds)], [(70, lds)]]
    assert [len(g["launches"]) for g in got] == [1, 1, 0, 1, 1, 1, 1, 1]
    assert got[2]["status"] != 0 and "product launch" in got[2]["error"]
    assert all(g["status"] == 0 for i, g in enumerate(got) if i != 2)
