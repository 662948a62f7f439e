"""The operators around the attention on the CPU: struct layouts, refusals
(status codes and messages, before anything is launched) and the rotation
frequencies."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _D():
    import paper_2609_03311_amd as D
    D.lib()
    return D


def test_struct_layouts_match_header(tmp_path):
    D = _D()
    structs = {"dopr_quantize_args_t": D._QuantizeArgs,
               "dopr_quant_matmul_args_t": D._QuantMatmulArgs,
               "dopr_norm_residual_args_t": D._NormResidualArgs,
               "dopr_rotary_args_t": D._RotaryArgs}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "dopr.h"',
             "int main(void) {"]
    for cname, py in structs.items():
        lines.append(f'printf("{cname} size %zu\\n", sizeof({cname}));')
        for f, _ in py._fields_:
            lines.append(f'printf("{cname} {f} %zu\\n", '
                         f'offsetof({cname}, {f}));')
    lines += ["return 0; }"]
    probe = tmp_path / "probe.c"
    probe.write_text("\n".join(lines))
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"),
                    str(probe), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True,
                         check=True).stdout
    got = {tuple(line.split()[:2]): int(line.split()[2])
           for line in out.splitlines()}
    for cname, py in structs.items():
        assert got[(cname, "size")] == ctypes.sizeof(py), cname
        for f, _ in py._fields_:
            assert got[(cname, f)] == getattr(py, f).offset, (cname, f)


def _fields(struct, **kw):
    a = struct()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _refused(D, fn, struct, good, bad, code, text):
    a = _fields(struct, **{**good, **bad})
    assert getattr(D.lib(), fn)(ctypes.byref(a), None) == code, bad
    assert text in D.dopr_last_error(), (bad, D.dopr_last_error())


# addresses are never dereferenced on the host
QUANT = dict(dtype=0, rows=4, width=64, x=256, x_row_stride=64, q=256,
             q_row_stride=64, scale=256)
MATMUL = dict(dtype=0, rows=4, cols=8, depth=64, x=256, x_row_stride=64,
              x_scale=256, w=256, w_row_stride=64, w_scale=256, y=256,
              y_row_stride=8)
NORM = dict(dtype=0, residual_dtype=0, rows=4, width=64, x=256,
            x_row_stride=64, residual_scale=1.0, rms_eps=1e-6, z=256,
            z_row_stride=64)
ROTARY = dict(dtype=0, n_q_heads=2, n_kv_heads=1, head_dim=64, rotary_dim=64,
              attention_factor=1.0, rms_eps=1e-6, rows=4, positions=256,
              inv_freq=256, q=256, q_row_stride=128, q_head_stride=64,
              q_out=256, q_out_row_stride=128, q_out_head_stride=64, k=256,
              k_row_stride=64, k_head_stride=64, k_out=256,
              k_out_row_stride=64, k_out_head_stride=64)

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -4


@pytest.mark.parametrize("bad,code,text", [
    (dict(dtype=3), INVALID, "dtype"),
    (dict(dtype=-1), INVALID, "dtype"),
    (dict(rows=-1), INVALID, "rows"),
    (dict(rows=1 << 31), INVALID, "rows"),
    (dict(width=0), INVALID, "width"),
    (dict(width=7), UNSUPPORTED, "width"),
    (dict(width=65537, x_row_stride=1 << 20, q_row_stride=1 << 20),
     UNSUPPORTED, "width"),
    (dict(x_row_stride=63), INVALID, "stride"),
    (dict(q_row_stride=0), INVALID, "stride"),
    (dict(up=256, up_row_stride=8), INVALID, "stride"),
    (dict(x=None), INVALID, "NULL"),
    (dict(scale=None), INVALID, "NULL"),
    (dict(x=257), INVALID, "aligned"),
    (dict(scale=258), INVALID, "aligned"),
    (dict(dtype=2, x=258), INVALID, "aligned"),
])
def test_quantize_refusals(bad, code, text):
    D = _D()
    _refused(D, "dopr_quantize_rows", D._QuantizeArgs, QUANT, bad, code, text)


@pytest.mark.parametrize("bad,code,text", [
    (dict(dtype=9), INVALID, "dtype"),
    (dict(rows=-1), INVALID, "rows"),
    (dict(cols=-5), INVALID, "cols"),
    (dict(depth=-1), INVALID, "depth"),
    (dict(depth=131072, x_row_stride=1 << 20, w_row_stride=1 << 20),
     UNSUPPORTED, "depth"),
    (dict(rows=(1 << 31) - 1, cols=(1 << 31) - 1), UNSUPPORTED, "blocks"),
    (dict(x_row_stride=63), INVALID, "stride"),
    (dict(w_row_stride=63), INVALID, "stride"),
    (dict(y_row_stride=7), INVALID, "stride"),
    (dict(residual=256, residual_row_stride=7), INVALID, "stride"),
    (dict(w=None), INVALID, "NULL"),
    (dict(w_scale=None), INVALID, "NULL"),
    (dict(y=257), INVALID, "aligned"),
    (dict(dtype=2, bias=258), INVALID, "aligned"),
    (dict(x_scale=258), INVALID, "aligned"),
])
def test_product_refusals(bad, code, text):
    D = _D()
    _refused(D, "dopr_quant_matmul", D._QuantMatmulArgs, MATMUL, bad, code,
             text)


@pytest.mark.parametrize("bad,code,text", [
    (dict(dtype=5), INVALID, "dtype"),
    (dict(residual_dtype=1), INVALID, "residual_dtype"),
    (dict(dtype=2, residual_dtype=0), INVALID, "residual_dtype"),
    (dict(width=4), UNSUPPORTED, "width"),
    (dict(residual_scale=float("nan")), INVALID, "residual_scale"),
    (dict(rms_eps=-1e-6), INVALID, "rms_eps"),
    (dict(rms_eps=float("inf")), INVALID, "rms_eps"),
    (dict(gate=256, gate_row_stride=32), INVALID, "stride"),
    (dict(residual=256, residual_row_stride=32), INVALID, "stride"),
    (dict(h=256, h_row_stride=32), INVALID, "stride"),
    (dict(z=None), INVALID, "no output"),
    (dict(q=256, q_row_stride=64), INVALID, "q_scale"),
    (dict(q_scale=256), INVALID, "q_scale"),
    (dict(x=None), INVALID, "NULL"),
    (dict(pre_norm_w=257), INVALID, "aligned"),
    (dict(residual_dtype=2, h=258, h_row_stride=64), INVALID, "aligned"),
])
def test_norm_refusals(bad, code, text):
    D = _D()
    _refused(D, "dopr_norm_residual", D._NormResidualArgs, NORM, bad, code,
             text)


@pytest.mark.parametrize("bad,code,text", [
    (dict(dtype=5), INVALID, "dtype"),
    (dict(n_q_heads=-1), INVALID, "heads"),
    (dict(rows=-2), INVALID, "rows"),
    (dict(rotary_dim=0), INVALID, "rotary_dim"),
    (dict(rotary_dim=33), INVALID, "rotary_dim"),
    (dict(rotary_dim=66), INVALID, "rotary_dim"),
    (dict(head_dim=514), UNSUPPORTED, "head_dim"),
    (dict(interleaved=2), INVALID, "interleaved"),
    (dict(inverse=1, q_norm_w=256), INVALID, "inverse"),
    (dict(attention_factor=float("inf")), INVALID, "attention_factor"),
    (dict(rms_eps=float("nan")), INVALID, "rms_eps"),
    (dict(positions=None), INVALID, "NULL"),
    (dict(k_out=None), INVALID, "NULL"),
    (dict(q_out_head_stride=32), INVALID, "overlap"),
    (dict(q_out_row_stride=64), INVALID, "overlap"),
    (dict(k_row_stride=-64), INVALID, "strides"),
    (dict(q=257), INVALID, "aligned"),
    (dict(inv_freq=258), INVALID, "aligned"),
])
def test_rotary_refusals(bad, code, text):
    D = _D()
    _refused(D, "dopr_rotary", D._RotaryArgs, ROTARY, bad, code, text)


def test_empty_calls_and_null_args():
    """No rows: OK without a launch, whatever the pointers."""
    D = _D()
    L = D.lib()
    for fn, struct, good in (
            ("dopr_quantize_rows", D._QuantizeArgs, QUANT),
            ("dopr_quant_matmul", D._QuantMatmulArgs, MATMUL),
            ("dopr_norm_residual", D._NormResidualArgs, NORM),
            ("dopr_rotary", D._RotaryArgs, ROTARY)):
        assert getattr(L, fn)(None, None) == INVALID
        assert "args is NULL" in D.dopr_last_error()
        a = _fields(struct, **{**good, "rows": 0})
        assert getattr(L, fn)(ctypes.byref(a), None) == D.DOPR_OK
    a = _fields(D._QuantMatmulArgs, **{**MATMUL, "cols": 0})
    assert L.dopr_quant_matmul(ctypes.byref(a), None) == D.DOPR_OK
    a = _fields(D._RotaryArgs, **{**ROTARY, "n_q_heads": 0, "n_kv_heads": 0})
    assert L.dopr_rotary(ctypes.byref(a), None) == D.DOPR_OK
    assert L.dopr_quant_matmul_workspace(ctypes.byref(a), None) == INVALID
    with pytest.raises(D.DoprError) as e:
        D.dopr_quant_matmul_workspace(4, 4, 131072)
    assert e.value.status == UNSUPPORTED


def test_product_workspace():
    """Sizes (both operands' rows at a pitch of whole spans of 128 bytes,
    none up to 16 rows or where 16 divides the depth) and its alignment."""
    D = _D()
    for m, n, k in ((1, 64, 100), (16, 64, 100), (129, 64, 4096),
                    (17, 0, 100), (17, 64, 0)):
        assert D.dopr_quant_matmul_workspace(m, n, k) == 0, (m, n, k)
    assert D.dopr_quant_matmul_workspace(17, 64, 100) == 81 * 128
    assert D.dopr_quant_matmul_workspace(1021, 2563, 2501) == 3584 * 2560
    _refused(D, "dopr_quant_matmul", D._QuantMatmulArgs, MATMUL,
             dict(workspace=128, workspace_bytes=4096), INVALID,
             "256-byte aligned")


def test_wrappers_refuse_wrong_tensors():
    """Types, shapes and devices are checked before pointers are taken."""
    D = _D()
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    q = torch.zeros(4, 64, dtype=torch.int8)
    s = torch.zeros(4)
    with pytest.raises(ValueError):
        D.dopr_quantize_rows(x, q, s)            # CPU tensors
    with pytest.raises(ValueError):
        D.dopr_quantize_rows(q, q, s)            # not a float type
    with pytest.raises(ValueError):
        D.dopr_quant_matmul(q, s, q, s, x)       # y is not [4, 4]
    with pytest.raises(ValueError):
        D.dopr_norm_residual(x, residual=x.half(), h=x)
    with pytest.raises(ValueError):
        D.dopr_rotary(None, None, s, s, None, None)


def test_rotary_frequencies():
    """Each scaling against its formula in 64 bits; fp32 rounding only."""
    D = _D()

    def check(got, ref):
        ref = np.asarray(ref)
        assert got.numpy().shape == ref.shape
        assert np.all(np.abs(got.numpy() - ref) <= 2.0 ** -24 * ref)

    for r, theta in ((128, 1e6), (64, 5e5), (6, 1e4), (2, 1e4)):
        i = np.arange(r // 2)
        w = theta ** (-2.0 * i / r)
        got, f = D.dopr_rotary_frequencies(r, theta)
        check(got, w)
        assert f == 1.0
        got, f = D.dopr_rotary_frequencies(r, theta, scaling="linear",
                                           factor=4)
        check(got, w / 4)
        for s, orig, lo, hi in ((4.0, 4096, 1, 32), (8.0, 8192, 1, 4),
                                (1.0, 2048, 2, 16)):
            kw = dict(factor=s, original_len=orig, turns_low=lo,
                      turns_high=hi)
            turns = orig * w / (2 * math.pi)
            g = np.clip((turns - lo) / (hi - lo), 0, 1)
            got, f = D.dopr_rotary_frequencies(r, theta, scaling="bands",
                                               **kw)
            check(got, w * (g + (1 - g) / s))
            assert f == 1.0
            # where the turns are met, as a real index
            at = [r * math.log(orig / (2 * math.pi * t)) /
                  (2 * math.log(theta)) for t in (lo, hi)]
            g = np.clip((at[0] - i) / (at[0] - at[1]), 0, 1)
            got, f = D.dopr_rotary_frequencies(r, theta, scaling="ramp", **kw)
            check(got, w * (g + (1 - g) / s))
            assert abs(f - (0.1 * math.log(s) + 1)) <= 1e-7
    got, _ = D.dopr_rotary_frequencies(64, 1e4, scaling="base", factor=8)
    # the fastest pair is kept, the slowest turns 8 times slower
    check(got[:1], [1.0])
    check(got[-1:], [1e4 ** (-62 / 64) / 8])
    bad = [dict(rotary_dim=0, theta=1e4), dict(rotary_dim=5, theta=1e4),
           dict(rotary_dim=64, theta=1.0),
           dict(rotary_dim=64, theta=float("inf")),
           dict(rotary_dim=64, theta=1e4, scaling="linear", factor=0.5),
           dict(rotary_dim=2, theta=1e4, scaling="base", factor=2),
           dict(rotary_dim=64, theta=1e4, scaling="ramp", factor=2),
           dict(rotary_dim=64, theta=1e4, scaling="bands", factor=2,
                original_len=4096, turns_low=4, turns_high=4)]
    for kw in bad:
        with pytest.raises(D.DoprError) as e:
            D.dopr_rotary_frequencies(**kw)
        assert e.value.status == D.DOPR_ERR_INVALID_ARG, kw
    with pytest.raises(ValueError):
        D.dopr_rotary_frequencies(64, 1e4, scaling="other")
