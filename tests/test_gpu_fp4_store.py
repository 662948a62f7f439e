"""A prefix store held in 4 bits: what goes in and comes out, bit for bit
against the format's definition in 64 bits, and every call that reads a store,
bit for bit against a bf16 store that holds the same values."""
import numpy as np
import pytest
import torch

import fp4_refs

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _D():
    import paper_2609_03311_amd as D
    return D


def _cu(lens):
    out = np.zeros(len(lens) + 1, np.int64)
    np.cumsum(lens, out=out[1:])
    return out


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _states(gen, rows, hkv, d, spread=False):
    """bf16 states on the CPU; spread: blocks of very different magnitudes,
    zeros and equal values among them."""
    x = torch.randn((rows, hkv, d), generator=gen)
    if spread and rows:
        x = x * torch.exp2(torch.randint(-40, 40, (rows, hkv, 1),
                                         generator=gen).float())
        x[torch.rand(rows, generator=gen) < 0.1] = 0.0
        x[torch.rand(rows, generator=gen) < 0.1] = -3.5
        x[..., :8] *= 2.0 ** -20
    return x.to(torch.bfloat16)


def _store(D, lens, hkv, d, fmt, layers=1):
    return D.dopr_store_create(layers, hkv, d, np.asarray(lens, np.int32),
                               format=fmt)


def _put(D, store, layer, ids, cu, k, v):
    D.dopr_store_put(store, layer, torch.tensor(ids, dtype=torch.int32,
                                                device=DEV),
                     torch.from_numpy(cu).to(DEV), k.to(DEV), v.to(DEV))


def _gather(D, store, layer, ids, cu, hkv, d):
    k, v = (torch.full((int(cu[-1]), hkv, d), 7.0, dtype=torch.bfloat16,
                       device=DEV) for _ in range(2))
    D.dopr_gather_prefix(store, layer,
                         torch.tensor(ids, dtype=torch.int32, device=DEV),
                         torch.from_numpy(cu).to(DEV), k, v)
    return k.cpu(), v.cpu()


def _same(a, b):
    """Equal bit for bit, any NaN for any NaN."""
    a, b = a.contiguous(), b.contiguous()
    nan = torch.isnan(a) & torch.isnan(b)
    return torch.equal(torch.where(nan, 0, a.view(torch.int16)),
                       torch.where(nan, 0, b.view(torch.int16)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv", [1, 3, 8, 11])
@pytest.mark.parametrize("spread", [False, True])
def test_put_and_gather(d, hkv, spread):
    D = _D()
    lens = [1, 0, 31, 32, 33, 64, 100, 5, 257]
    cu = _cu(lens)
    k, v = (_states(_gen(s + hkv), int(cu[-1]), hkv, d, spread)
            for s in (1, 2))
    store = _store(D, lens, hkv, d, D.DOPR_STORE_FP4, layers=2)
    ids = list(range(len(lens)))
    _put(D, store, 0, ids, cu, v, k)
    _put(D, store, 1, ids, cu, k, v)
    for layer, (a, b) in ((1, (k, v)), (0, (v, k))):
        want = fp4_refs.held(a, b, cu)
        got = _gather(D, store, layer, ids, cu, hkv, d)
        assert _same(got[0], want[0]) and _same(got[1], want[1])
    assert D.dopr_check_status(store) == D.DOPR_OK


def test_held_values_stay_what_they_are():
    """Putting what came out of a store changes nothing."""
    D = _D()
    lens, hkv, d = [70, 33], 2, 128
    cu = _cu(lens)
    k, v = (_states(_gen(s), int(cu[-1]), hkv, d, True) for s in (3, 4))
    store = _store(D, lens, hkv, d, D.DOPR_STORE_FP4)
    _put(D, store, 0, [0, 1], cu, k, v)
    first = _gather(D, store, 0, [0, 1], cu, hkv, d)
    _put(D, store, 0, [0, 1], cu, *first)
    again = _gather(D, store, 0, [0, 1], cu, hkv, d)
    assert _same(first[0], again[0]) and _same(first[1], again[1])


def test_ends_of_the_range():
    """Zeros of either sign, the smallest and largest bf16 values, blocks with
    infinities and NaN."""
    D = _D()
    lens, hkv, d = [65], 1, 64
    cu = _cu(lens)
    k, v = (_states(_gen(s), 65, hkv, d) for s in (5, 6))
    for x in (k, v):
        x[0] = -0.0
        x[1] = 2.0 ** -133
        x[2, 0, ::2] = 2.0 ** -126
        x[3] = 3.3895e38
        x[4, 0, 5] = float("inf")
        x[5, 0, 9] = float("-inf")
        x[6, 0, 17] = float("nan")
        x[40:, :, 3] = 1e-30
    store = _store(D, lens, hkv, d, D.DOPR_STORE_FP4)
    _put(D, store, 0, [0], cu, k, v)
    want = fp4_refs.held(k, v, cu)
    got = _gather(D, store, 0, [0], cu, hkv, d)
    assert torch.isnan(want[0]).sum() == 3 * 32
    assert _same(got[0], want[0]) and _same(got[1], want[1])


def test_bad_documents_are_skipped():
    D = _D()
    lens, hkv, d = [4, -1, 40], 2, 64
    cu = _cu([4, 4, 39, 4, 40])
    k, v = (_states(_gen(s), int(cu[-1]), hkv, d) for s in (7, 8))
    store = _store(D, lens, hkv, d, D.DOPR_STORE_FP4)
    _put(D, store, 0, [0, 1, 2, 9, 2], cu, k, v)
    assert D.dopr_check_status(store) == D.DOPR_ERR_DOC_RANGE
    wk, wv = fp4_refs.held(k, v, cu)
    got = _gather(D, store, 0, [2, 1, 0], _cu([40, 4, 4]), hkv, d)
    assert D.dopr_check_status(store) == D.DOPR_ERR_DOC_RANGE
    for g, w in zip(got, (wk, wv)):
        assert _same(g[:40], w[-40:]) and _same(g[44:], w[:4])
        assert (g[40:44] == 7.0).all()


def test_copy_docs():
    D = _D()
    lens, hkv, d = [33, 8, 64, -1], 3, 128
    cu = _cu(lens[:3])
    k, v = (_states(_gen(s), int(cu[-1]), hkv, d) for s in (9, 10))
    src = _store(D, lens, hkv, d, D.DOPR_STORE_FP4, layers=2)
    for layer in (0, 1):
        _put(D, src, layer, [0, 1, 2], cu, k, v)
    dst = _store(D, [33, -1, 64, 5], hkv, d, D.DOPR_STORE_FP4, layers=2)
    D.dopr_store_copy_docs(dst, src)
    wk, wv = fp4_refs.held(k, v, cu)
    got = _gather(D, dst, 1, [2, 0], _cu([64, 33]), hkv, d)
    for g, w in zip(got, (wk, wv)):
        assert _same(g[:64], w[41:]) and _same(g[64:], w[:33])
    assert D.dopr_check_status(dst) == D.DOPR_OK
    other = _store(D, lens, hkv, d, D.DOPR_STORE_BF16, layers=2)
    for a, b in ((other, src), (src, other)):
        with pytest.raises(D.DoprError) as e:
            D.dopr_store_copy_docs(a, b)
        assert e.value.status == D.DOPR_ERR_INVALID_ARG


# ---------------------------------------------------------------------------
# Keys normed and turned on the way in

def _expected(k, v, cu, fmt, D, **kw):
    k = fp4_refs.turned_keys(k, **kw)
    v = v.to(torch.bfloat16)
    return (k, v) if fmt == D.DOPR_STORE_BF16 else fp4_refs.held(k, v, cu)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16,
                                   torch.float32])
@pytest.mark.parametrize("d,rotated,inter", [
    (128, 128, False), (128, 128, True), (128, 64, False), (128, 50, False),
    (128, 2, True), (64, 64, False), (64, 16, True), (64, 30, False)])
def test_put_rotary(fmt, dtype, d, rotated, inter):
    D = _D()
    lens, hkv = [1, 0, 40, 100, 32], 3
    cu = _cu(lens)
    rows = int(cu[-1])
    gen = _gen(rotated + d)
    # k and v parts of one buffer's rows that start at an odd element
    buf = torch.randn((rows, 1 + (4 + 2 * hkv) * d), generator=gen).to(dtype)
    k = buf[:, 1 + 4 * d:1 + (4 + hkv) * d].unflatten(1, (hkv, d))
    v = buf[:, 1 + (4 + hkv) * d:].unflatten(1, (hkv, d))
    gain = (1 + 0.1 * torch.randn(d, generator=gen)).to(dtype)
    pos = torch.randint(0, 100000, (rows,), generator=gen, dtype=torch.int32)
    freq = 1e6 ** (-torch.arange(0, rotated, 2) / rotated)
    ids = torch.arange(len(lens), dtype=torch.int32)
    on = buf.to(DEV)
    kd = on[:, 1 + 4 * d:1 + (4 + hkv) * d].unflatten(1, (hkv, d))
    vd = on[:, 1 + (4 + hkv) * d:].unflatten(1, (hkv, d))
    for g, p, factor in ((gain, pos, 1.25), (None, pos, 1.0), (gain, None,
                                                              1.0)):
        store = _store(D, lens, hkv, d, fmt)
        D.dopr_store_put_rotary(
            store, 0, ids.to(DEV), torch.from_numpy(cu).to(DEV), kd, vd,
            freq.to(DEV), positions=None if p is None else p.to(DEV),
            k_norm_w=None if g is None else g.to(DEV), interleaved=inter,
            attention_factor=factor)
        if p is None:
            p = torch.cat([torch.arange(n) for n in lens])
        want = _expected(k, v, cu, fmt, D, positions=p, inv_freq=freq,
                         gain=g, interleaved=inter, factor=factor)
        got = _gather(D, store, 0, ids.tolist(), cu, hkv, d)
        assert _same(got[0], want[0]) and _same(got[1], want[1])


def test_put_rotary_head_major():
    """Heads further apart than rows, and rows a document's put does not
    name."""
    D = _D()
    lens, hkv, d = [50, 20], 4, 64
    rows = 90
    k, v = (torch.randn((hkv, rows, d), generator=_gen(s)).transpose(0, 1)
            for s in (11, 12))
    freq = 1e4 ** (-torch.arange(0, d, 2) / d)
    for fmt in (0, 1):
        store = _store(D, lens, hkv, d, fmt)
        cu = np.array([10, 60, 80], np.int64)
        D.dopr_store_put_rotary(
            store, 0, torch.tensor([0, 1], dtype=torch.int32, device=DEV),
            torch.from_numpy(cu).to(DEV), k.to(DEV), v.to(DEV),
            freq.to(DEV))
        p = torch.cat([torch.arange(50), torch.arange(20)])
        want = _expected(k[10:80], v[10:80], cu - 10, fmt, D, positions=p,
                         inv_freq=freq)
        got = _gather(D, store, 0, [0, 1], cu - 10, hkv, d)
        assert _same(got[0], want[0]) and _same(got[1], want[1])


def test_put_rotary_rows_outside_the_source():
    """A document whose rows lie outside k and v is reported, not read."""
    D = _D()
    store = _store(D, [4, 4], 1, 64, 1)
    k = torch.ones((8, 1, 64), device=DEV)
    freq = torch.ones(32, device=DEV)
    ids = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    for cu in ([-2, 2, 6], [2, 6, 10]):
        D.dopr_store_put_rotary(store, 0, ids,
                                torch.tensor(cu, device=DEV), k, k, freq)
        assert D.dopr_check_status(store) == D.DOPR_ERR_DOC_RANGE


@pytest.mark.parametrize("fmt", [0, 1])
def test_angles_of_any_size(fmt):
    """Positions of either sign up to the type's ends, and frequencies past
    any model's."""
    D = _D()
    lens, hkv, d = [70], 2, 64
    cu = _cu(lens)
    k, v = (torch.randn((70, hkv, d), generator=_gen(s)) for s in (21, 22))
    pos = torch.randint(-2 ** 31, 2 ** 31, (70,), generator=_gen(23),
                        dtype=torch.int64).to(torch.int32)
    pos[:3] = torch.tensor([2 ** 31 - 1, -2 ** 31, 0])
    freq = 10.0 ** torch.linspace(-12, 9, d // 2)
    store = _store(D, lens, hkv, d, fmt)
    D.dopr_store_put_rotary(
        store, 0, torch.zeros(1, dtype=torch.int32, device=DEV),
        torch.from_numpy(cu).to(DEV), k.to(DEV), v.to(DEV), freq.to(DEV),
        positions=pos.to(DEV))
    want = _expected(k, v, cu, fmt, D, positions=pos, inv_freq=freq)
    got = _gather(D, store, 0, [0], cu, hkv, d)
    assert _same(got[0], want[0]) and _same(got[1], want[1])
