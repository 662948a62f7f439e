"""The 4-bit prefix store on the CPU: sizes, struct layout, refusals and
launches."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from store_calls import store_calls

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -4


def _D():
    import paper_2609_03311_amd as D
    D.lib()
    return D


def test_store_bytes_closed_form():
    D = _D()
    rng = np.random.default_rng(0)
    for layers, hkv, d in [(1, 8, 128), (36, 8, 128), (3, 2, 64)]:
        lens = rng.integers(-1, 300, 500).astype(np.int32)
        pool, payload = D.dopr_store_bytes(layers, hkv, d, lens,
                                           D.DOPR_STORE_FP4)
        n = lens[lens >= 0].astype(np.int64)
        chunks = -(-n // 32)
        # half a byte a value of K and V, a byte for 32 dims of a key and for
        # a chunk's slots of a value's dim
        assert payload == layers * hkv * (n * d + n * (d // 32)
                                          + chunks * d).sum()
        index = (12 + 4 * layers * hkv) * len(lens)
        held = 34 * d * chunks.sum() * layers * hkv
        assert held + index <= pool <= held + index + 5 * 256
        assert (pool, payload) == D.dopr_store_bytes_as(layers, hkv, d, lens,
                                                        D.DOPR_STORE_FP4)
        assert D.dopr_store_bytes_as(layers, hkv, d, lens,
                                     D.DOPR_STORE_BF16) == \
            D.dopr_store_bytes(layers, hkv, d, lens)


def test_store_refusals():
    D = _D()
    for fmt in (-1, 2):
        with pytest.raises(D.DoprError) as e:
            D.dopr_store_bytes(1, 8, 128, [4], fmt)
        assert e.value.status == INVALID and "format" in str(e.value)
    with pytest.raises(D.DoprError) as e:
        D.dopr_store_bytes(1, 8, 96, [4], D.DOPR_STORE_FP4)
    assert e.value.status == UNSUPPORTED
    for longest, good in ((2 ** 31 - 64, True), (2 ** 31 - 63, False)):
        if good:
            assert D.dopr_store_bytes(1, 1, 64, [longest],
                                      D.DOPR_STORE_FP4)[0] > 68 * longest
            continue
        with pytest.raises(D.DoprError) as e:
            D.dopr_store_bytes(1, 1, 64, [longest], D.DOPR_STORE_FP4)
        assert e.value.status == UNSUPPORTED
    L = D.lib()
    desc, _keep = D._desc(1, 8, 128, [4])
    h = ctypes.c_void_p(0)
    pool, _ = D.dopr_store_bytes(1, 8, 128, [4], D.DOPR_STORE_FP4)
    for at, size, code in ((None, pool, INVALID), (128, pool, INVALID),
                           (256, pool - 1, WORKSPACE)):
        assert L.dopr_store_create_as(ctypes.byref(desc), 1, at, size, None,
                                      ctypes.byref(h)) == code
    assert L.dopr_store_create_as(ctypes.byref(desc), 7, 256, pool, None,
                                  ctypes.byref(h)) == INVALID
    assert L.dopr_store_put_rotary(None, None, None) == INVALID


def test_struct_layout_matches_header(tmp_path):
    D = _D()
    py, cname = D._PutRotaryArgs, "dopr_put_rotary_args_t"
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "dopr.h"',
             "int main(void) {", f'printf("%zu\\n", sizeof({cname}));']
    lines += [f'printf("%zu\\n", offsetof({cname}, {f}));'
              for f, _ in py._fields_]
    probe = tmp_path / "probe.c"
    probe.write_text("\n".join(lines + ["return 0; }"]))
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"),
                    str(probe), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True,
                         check=True).stdout.split()
    assert [int(x) for x in out] == [ctypes.sizeof(py)] + [
        getattr(py, f).offset for f, _ in py._fields_]


PUT = dict(layer=0, dtype=0, n=2, rows=100, doc_ids=256, src_cu_slots=256,
           k=256, k_row_stride=256, k_head_stride=128, v=256,
           v_row_stride=256, v_head_stride=128, inv_freq=256, rotary_dim=128,
           attention_factor=1.0, rms_eps=1e-6)


def _put(**more):
    return ["dopr_store_put_rotary", "_PutRotaryArgs", PUT | more]


def test_put_rotary_refusals():
    bad = [(dict(layer=2), "layer"), (dict(layer=-1), "layer"),
           (dict(dtype=3), "dtype"), (dict(n=-1), "bad n"),
           (dict(n=1 << 31), "bad n"), (dict(rows=-1), "rows"),
           (dict(rotary_dim=0), "rotary_dim"),
           (dict(rotary_dim=7), "rotary_dim"),
           (dict(rotary_dim=130), "rotary_dim"),
           (dict(interleaved=2), "interleaved"),
           (dict(attention_factor=float("inf")), "attention_factor"),
           (dict(rms_eps=-1.0), "rms_eps"),
           (dict(rms_eps=float("nan")), "rms_eps"),
           (dict(k_row_stride=-1), "strides"),
           (dict(v_head_stride=-1), "strides"), (dict(k=None), "NULL"),
           (dict(v=None), "NULL"), (dict(doc_ids=None), "NULL"),
           (dict(src_cu_slots=None), "NULL"), (dict(inv_freq=None), "NULL"),
           (dict(k=257), "aligned"), (dict(dtype=2, v=258), "aligned"),
           (dict(k_norm_w=255), "aligned"), (dict(positions=258), "aligned"),
           (dict(inv_freq=258), "aligned"),
           (dict(src_cu_slots=260), "aligned")]
    for fmt in (0, 1):
        got = store_calls((2, 2, 128, [5, 6], fmt),
                          [_put(**b) for b, _ in bad])
        for (b, text), g in zip(bad, got):
            assert g["status"] == INVALID and not g["launches"], b
            assert text in g["error"], (b, g)


def test_put_launches():
    got = store_calls((1, 2, 64, [40, 300], 1), [
        _put(n=0, rotary_dim=64), _put(rotary_dim=64),
        _put(n=(1 << 23) + 5, rotary_dim=64),
        ["dopr_store_put", None, [0, 1, 256, 256, 256, 256]],
        ["dopr_gather_prefix", None, [0, 1, 256, 256, 256, 256]],
        ["dopr_gather_prefix", None, [0, (1 << 24) + 1, 256, 256, 256, 256]],
    ])
    assert all(g["status"] == 0 for g in got)
    names = [[x["kernel"].split("<")[0] for x in g["launches"]] for g in got]
    assert names[0] == []
    # ten chunks of the longest document in blocks of their own, their key
    # bounds cleared in front
    assert names[1] == ["k_put_clear", "k_put_states"]
    assert (got[1]["launches"][1]["gx"], got[1]["launches"][1]["gy"]) == \
        (2, 10)
    # (the last slice's five documents' chunks again)
    assert names[2] == ["k_put_states"] + ["k_put_clear", "k_put_states"]
    assert names[3] == ["k_put_clear", "k_put_states"]
    assert names[4] == ["k_gather_fp4"] and names[5] == ["k_gather_fp4"] * 3
    for g in got:
        for x in g["launches"]:
            assert x["gx"] * x["bx"] < 1 << 32 and x["gy"] <= 65535


ATTN = dict(_layer=0, n_pairs=1, n_q_heads=8, max_tokens=1, total_tokens=1,
            doc_ids=256, cu_seqlens=256, q=256, k=256, v=256, rms_eps=1e-6,
            rope_theta=1e6, softmax_scale=0.1, out=256, workspace=256,
            workspace_bytes=1 << 60)


def _attn(**more):
    return ["dopr_prefix_attn", "_AttnArgs", ATTN | more]


def _kernels(got):
    for g in got:
        assert g["status"] == 0, g["error"]
        for x in g["launches"]:
            assert x["gx"] * x["bx"] < 1 << 32 and x["gy"] <= 65535, x
            assert x["lds"] <= 160 << 10
    return [[x["kernel"].split("<")[0] for x in g["launches"]] for g in got]


@pytest.mark.parametrize("d", [64, 128])
def test_attention_launches(d):
    """Which kernels a call over a 4-bit store takes by itself, and their
    grids at its largest."""
    short = _kernels(store_calls((1, 2, d, [40, 300], 1), [
        _attn(), _attn(n_pairs=5000, total_tokens=5000),
        # a pair without the one token it has to have is not for them
        _attn(max_tokens=2, total_tokens=2),
        _attn(n_pairs=64, max_tokens=90, total_tokens=64 * 90),
        _attn(n_pairs=0, max_tokens=5, total_tokens=0),
        _attn(n_pairs=(1 << 24) + 3, total_tokens=(1 << 24) + 3),
        _attn(n_pairs=(1 << 24) + 3, max_tokens=9, total_tokens=1 << 26),
    ]))
    rows = ["k_own_keys", "k_rows_fp4"]
    assert short[:5] == [["k_token_fp4"], ["k_token_fp4"], rows, rows, []]
    assert set(short[5]) == {"k_token_fp4"} and set(short[6]) == set(rows)
    long = _kernels(store_calls((1, 2, d, [40, 60000], 1), [
        _attn(), _attn(max_tokens=2, total_tokens=2),
        _attn(n_pairs=5000, total_tokens=5000),
        _attn(n_pairs=64, max_tokens=90, total_tokens=64 * 90)]))
    assert long == [["k_token_fp4", "k_token_join"], rows + ["k_rows_join"],
                    ["k_token_fp4"], rows]
    # the planned kernels where they are asked for
    for variant, name in ((8, "k_pass_attn"), (6, "k_prefix_attn"),
                          (1, "k_prefix_attn"), (4, "k_prefix_attn")):
        got = _kernels(store_calls((1, 2, d, [40, 300], 1), [
            _attn(n_pairs=5, max_tokens=9, total_tokens=45,
                  kernel_variant=variant)]))
        assert name in got[0] and not set(got[0]) & set(rows), variant


def test_attention_refusals():
    D = _D()
    doc_len = [40, 60000]
    pool, _ = D.dopr_store_bytes(1, 2, 128, doc_len, D.DOPR_STORE_FP4)
    desc, _keep = D._desc(1, 2, 128, doc_len)
    shapes = [dict(), dict(max_tokens=5, total_tokens=5),
              dict(n_pairs=900, max_tokens=50, total_tokens=45000)]
    bad = [(dict(workspace_bytes=255), "workspace"),
           (dict(workspace=257), "aligned"), (dict(workspace=None), ""),
           (dict(q=None), "NULL"), (dict(doc_ids=None), "NULL"),
           (dict(q=260), "aligned"), (dict(out=264), "aligned"),
           (dict(n_q_heads=7), "n_q_heads"),
           (dict(q_norm_w=256), "norm"), (dict(softmax_scale=0.0), "scale"),
           (dict(softmax_scale=float("nan")), "scale"),
           (dict(rms_eps=float("nan")), "rms_eps"),
           (dict(kernel_variant=7), "kernel_variant"),
           (dict(max_tokens=0), "max_tokens"), (dict(_layer=1), "layer"),
           (dict(_layer=-1), "layer"), (dict(rope_inv_freq=258), "aligned")]
    for shape in shapes:
        got = store_calls((1, 2, 128, doc_len, 1),
                          [_attn(**{**shape, **b}) for b, _ in bad])
        for (b, text), g in zip(bad, got):
            if b == dict(workspace_bytes=255) and not shape:
                continue  # (may need less)
            assert g["status"] in (INVALID, WORKSPACE), (b, g)
            assert not g["launches"] and text in g["error"], (b, g)


def test_put_rotary_checks_its_tensors():
    """The binding names the argument; nothing of a CPU tensor reaches the
    library."""
    import torch
    D = _D()

    class Stand:
        handle, n_kv_heads, head_dim = 0, 2, 64
        pool = torch.empty(0)

    k = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    ids = torch.zeros(1, dtype=torch.int32)
    cu = torch.tensor([0, 5])
    freq = torch.ones(32)
    good = [ids, cu, k, k, freq]
    for i, what in enumerate(("doc_ids", "src_cu_slots", "k", "v",
                              "inv_freq")):
        for wrong in (None, 3, torch.zeros(2, 3, dtype=torch.int16)):
            args = list(good)
            args[i] = wrong
            with pytest.raises(ValueError):
                D.dopr_store_put_rotary(Stand(), 0, *args)
    with pytest.raises(ValueError, match="k must be a"):
        D.dopr_store_put_rotary(Stand(), 0, *good)  # (on the CPU)
    with pytest.raises(ValueError, match="kv heads"):
        D.dopr_store_put_rotary(Stand(), 0, ids, cu, k.flatten(1), k, freq)
