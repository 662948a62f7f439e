"""The operators' sources and launches, looked at on the host (no GPU)."""
import os
import subprocess

import pytest

from operator_launches import kernels, launches
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


MANY = 1 << 31


def rows_call(rows, width):
    return ["dopr_quantize_rows", "_QuantizeArgs",
            dict(dtype=1, rows=rows, width=width, x=256, x_row_stride=width,
                 q=256, q_row_stride=width, scale=256)]


def norm_call(rows, width):
    return ["dopr_norm_residual", "_NormResidualArgs",
            dict(dtype=0, residual_dtype=2, rows=rows, width=width, x=256,
                 x_row_stride=width, residual_scale=1.0, rms_eps=1e-6, h=256,
                 h_row_stride=width, z=256, z_row_stride=width)]


def rotary_call(rows, heads, dim):
    pitch = heads * dim
    return ["dopr_rotary", "_RotaryArgs",
            dict(dtype=0, n_q_heads=heads, n_kv_heads=0, head_dim=dim,
                 rotary_dim=dim, attention_factor=1.0, rms_eps=1e-6,
                 rows=rows, positions=256, inv_freq=256, q=256,
                 q_row_stride=pitch, q_head_stride=dim, q_out=256,
                 q_out_row_stride=pitch, q_out_head_stride=dim)]


# (call, items, items a block takes): every row, token, strip of 16 columns,
# tile or piece of 16 bytes belongs to one block
LARGE = [
    (rows_call(MANY - 1, 8), MANY - 1, 4),
    (rows_call((1 << 26) - 4, 8), (1 << 26) - 4, 4),
    (rows_call(1 << 26, 2048), 1 << 26, 4),
    (rows_call(1 << 25, 4096), 1 << 25, 1),
    (rows_call(1 << 23, 65536), 1 << 23, 1),
    (norm_call(MANY - 1, 8), MANY - 1, 4),
    (norm_call(1 << 24, 4096), 1 << 24, 1),
    (norm_call((1 << 22) + 1, 65000), (1 << 22) + 1, 1),
    (rotary_call(MANY - 1, 1, 64), MANY - 1, 4),
    (rotary_call((1 << 26) + 3, 3, 512), (1 << 26) + 3, 4),
    (product(1, MANY - 1025, 16), -(-(MANY - 1025) // 16), 1),
    (product(16, 1 << 28, 1), 1 << 24, 1),
    (product(MANY - 1025, 1, 1, x_row_stride=1), -(-(MANY - 1025) // 64), 1),
    (product(17, MANY - 1025, 1, x_row_stride=1, w_row_stride=1),
     -(-(MANY - 1025) // 128), 1),
    (product(1 << 29, 65, 1, x_row_stride=1, w_row_stride=1,
             workspace=256, workspace_bytes=(1 << 29) * 128 + 65 * 128),
     (1 << 32) + 520, 256),
]


def test_launches_of_many_rows_fit():
    """Sizes whose rows ask for 2^32 threads and more come as several
    launches (one has fewer), every row, token or column in one of them;
    tiles that a block takes in turn need no more than fill the GPU."""
    for (_, items, per), got in zip(LARGE, launches([c for c, _, _ in LARGE])):
        assert got["status"] == 0, got["error"]
        run = [k for k in got["launches"] if not k["kernel"].startswith(
            "k_product<")]
        for k in got["launches"]:
            assert k["gx"] * k["bx"] < 1 << 32 and k["gy"] * k["gz"] < 1 << 16
        blocks = sum(k["gx"] for k in run)
        least = -(-items // per)
        assert least <= blocks < least + len(run), (got, items)


def test_ordinary_calls_are_one_launch():
    for call in (rows_call(12900, 12288), norm_call(20011, 2561),
                 rotary_call(32768, 40, 128), product(1, 6144, 4096),
                 product(12900, 24576, 4096),
                 product(600, 520, 777, x_row_stride=777)):
        got, = launches([call])
        assert got["status"] == 0 and len(got["launches"]) == 1


@pytest.mark.parametrize("how,needs", [
    (dict(), False),                                   # sizes alone
    (dict(x=256, w=512, x_row_stride=4096, w_row_stride=4096), False),
    (dict(x=257), True),
    (dict(w=264), True),
    (dict(x_row_stride=4100), True),
    (dict(w_row_stride=4104), True),
    (dict(w_row_stride=1 << 22), True),                # past 32-bit offsets
    (dict(depth=4090), True),
    (dict(depth=4090, x_row_stride=4096), True),       # w's back to back
    (dict(depth=4090, x_row_stride=4096, w_row_stride=4112), False),
    (dict(depth=0, x=257), False),
    (dict(rows=16, x=257), False),
    (dict(cols=0, x=257), False),
])
def test_workspace_is_asked_for_where_it_is_used(how, needs):
    """The bytes asked for are those a call with such rows uses: with them
    rows are laid out again, without any they are multiplied as they lie, and
    where none are asked for neither happens."""
    import ctypes

    import paper_2609_03311_amd as D
    a = D._QuantMatmulArgs()
    fields = dict(rows=200, cols=300, depth=4096) | how
    for k, v in fields.items():
        setattr(a, k, v)
    n = ctypes.c_size_t(7)
    assert D.lib().dopr_quant_matmul_workspace(
        ctypes.byref(a), ctypes.byref(n)) == 0
    rows = (fields["rows"] + fields["cols"]) * 4096
    assert n.value == (rows if needs else 0)
    if fields["depth"] == 0 or fields["cols"] == 0:
        return
    k = fields["depth"]
    call = product(**fields | dict(x_row_stride=how.get("x_row_stride", k),
                                   w_row_stride=how.get("w_row_stride", k)))
    call[2] |= dict(x=how.get("x", 256), w=how.get("w", 256))
    with_it = [call[0], call[1],
               call[2] | dict(workspace=256, workspace_bytes=n.value)]
    names = [[k["kernel"] for k in g["launches"]]
             for g in launches([call, with_it])]
    if needs:
        assert names[0] == ["k_product_any<bf16_t>"]
        assert names[1][0] == "k_repack" and len(names[1]) == 2
    else:
        assert names[0] == names[1] and "any" not in names[0][0]


def test_workspace_by_tensors():
    import torch

    import paper_2609_03311_amd as D
    x = torch.zeros(200, 4112, dtype=torch.int8)
    w = torch.zeros(300, 4096, dtype=torch.int8)
    size = 500 * 4096
    assert x.data_ptr() % 16 == w.data_ptr() % 16 == 0
    assert D.dopr_quant_matmul_workspace(200, 300, 4096) == 0
    assert D.dopr_quant_matmul_workspace(200, 300, 4096, x=x[:, 1:4097],
                                         w=w) == size
    assert D.dopr_quant_matmul_workspace(200, 300, 4080, x=x[:, :4080],
                                         w=w[:, :4080]) == 0
    assert D.dopr_quant_matmul_workspace(200, 300, 4090) == size
    assert D.dopr_quant_matmul_workspace(200, 300, 4090, x=x[:, :4090],
                                         w=w[:, :4090]) == 0


def test_flags_without_a_truth_value_are_refused():
    import numpy as np
    import torch

    import paper_2609_03311_amd as D
    x = torch.zeros(4, 2, 64)
    f = torch.zeros(32)
    p = torch.zeros(4, dtype=torch.int32)
    for flag in ("interleaved", "inverse"):
        with pytest.raises(ValueError, match="ambiguous"):
            D.dopr_rotary(x, None, p, f, x, None,
                          **{flag: np.array([True, False])})


def product_way(call, got):
    """How a call of rows on 16-byte addresses runs: its kernel, how many
    tiles a block takes (3: more than two), whether the depth ends in a
    partial span, and whether it is shorter than the spans in flight."""
    k, = got["launches"]
    name = k["kernel"]
    if not name.startswith("k_product<"):
        return name, 1, False, False
    fm, wgm, wgn, wk, st = map(int, name[:-1].split(",")[1:])
    a = call[2]
    tiles = -(-a["rows"] // (16 * fm * wgm)) * -(-a["cols"] // (64 * wgn))
    return (name, min(-(-tiles // k["gx"]), 3), a["depth"] % 128 > 0,
            a["depth"] // 128 // wk < st)


def test_gpu_tests_reach_every_way_a_product_runs():
    """Whatever way random sizes take is taken by one of the sizes that the
    GPU tests compare bit for bit: costs that are fitted anew may pick other
    kernels, and then more sizes have to be listed."""
    import math
    import random

    from product_sizes import SIZES
    calls = [product(*size) for size in SIZES]
    covered = {product_way(c, g) for c, g in zip(calls, launches(calls))}
    rng = random.Random(5)

    def size(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    sizes = [(size(1, 9000), size(32, 60000), size(20, 9000))
             for _ in range(8000)]
    calls = [product(m, n, k if i % 2 else -(-k // 128) * 128)
             for i, (m, n, k) in enumerate(sizes) if m * n < 9e7]
    missed = {}
    for c, g in zip(calls, launches(calls)):
        missed.setdefault(product_way(c, g), c[2])
    missed = {w: [c[k] for k in ("rows", "cols", "depth")]
              for w, c in missed.items() if w not in covered}
    assert not missed
    # and every kernel that is compiled for such rows
    names = {w[0] for w in covered}
    compiled = {n for n in kernels() if n.startswith("k_product") and
                "<bf16_t" in n and "any" not in n}
    assert names == compiled
