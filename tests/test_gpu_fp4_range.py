"""Keys over their type's whole range on their way into a store, normed and
turned, bit for bit against the 64-bit form (rounded to fp32 and from there to
bf16, as the store takes them)."""
import pytest
import torch

from test_gpu_fp4_store import _cu, _expected, _gather, _gen, _same, _store
from test_gpu_operators_range import EXPONENTS

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _D():
    import paper_2609_03311_amd as D
    return D


def _scaled(x, exponents):
    return torch.ldexp(x.double(), torch.tensor(exponents).double().view(
        -1, *[1] * (x.dim() - 1)))


def _check(k, gain, d, rotated, inter, eps, factor=1.0):
    """k [rows, Hkv, D] (CPU) into stores of both formats, as two documents."""
    D = _D()
    rows, hkv = k.shape[:2]
    lens = [rows - rows // 3, rows // 3]
    cu = _cu(lens)
    v = torch.randn(k.shape, generator=_gen(1)).to(k.dtype)
    pos = torch.randint(0, 5000, (rows,), generator=_gen(2),
                        dtype=torch.int32)
    freq = 1e4 ** (-torch.arange(0, rotated, 2) / rotated)
    for fmt in (D.DOPR_STORE_BF16, D.DOPR_STORE_FP4):
        store = _store(D, lens, hkv, d, fmt)
        D.dopr_store_put_rotary(
            store, 0, torch.tensor([0, 1], dtype=torch.int32, device=DEV),
            torch.from_numpy(cu).to(DEV), k.to(DEV), v.to(DEV), freq.to(DEV),
            positions=pos.to(DEV), interleaved=inter, rms_eps=eps,
            attention_factor=factor,
            k_norm_w=None if gain is None else gain.to(DEV))
        want = _expected(k, v, cu, fmt, D, positions=pos, inv_freq=freq,
                         gain=gain, interleaved=inter, eps=eps,
                         factor=factor)
        got = _gather(D, store, 0, [0, 1], cu, hkv, d)
        assert _same(got[0], want[0]) and _same(got[1], want[1]), fmt


ROTATIONS = [(128, 128, False), (128, 64, False), (128, 50, False),
             (128, 128, True), (64, 64, False), (64, 16, True)]


@pytest.mark.parametrize("eps", [0.0, 1e-36, 1e-6])
@pytest.mark.parametrize("d,rotated,inter", ROTATIONS)
@pytest.mark.parametrize("dtype", list(EXPONENTS))
def test_keys_of_any_size(dtype, d, rotated, inter, eps):
    """Rows of every size side by side, with gains about one, and without a
    norm (sums next to the type's end may pass it)."""
    e = EXPONENTS[dtype] * 3
    gen = _gen(d + rotated)
    k = _scaled(torch.randn((len(e), 3, d), generator=gen), e).to(dtype)
    gain = (1 + 0.1 * torch.randn(d, generator=gen)).to(dtype)
    for g in (gain, None):
        _check(k, g, d, rotated, inter, eps)


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("d,rotated,inter", ROTATIONS)
def test_products_with_gains_that_leave_fp32(d, rotated, inter, eps):
    """A bf16 value times a bf16 gain has fp32's bits, not its range: rows at
    the type's ends, gains of any size."""
    gen = _gen(3)
    e = [-133, -126, -120, -100, 0, 100, 120, 126] * 5
    k = _scaled(torch.randn((len(e), 2, d), generator=gen), e)
    k = k.clamp(-3.3895e38, 3.3895e38).to(torch.bfloat16)
    k[3::8] = 3.0e38
    k[4::8, 1] = torch.finfo(torch.bfloat16).max
    about_one = 1 + 0.1 * torch.randn(d, generator=gen)
    spread = torch.randint(-30, 30, (d,), generator=gen).double()
    for gain in (torch.full((d,), 1.25), 40 * about_one, about_one * 2e-30,
                 torch.ldexp(about_one.double(), spread)):
        _check(k, gain.to(torch.bfloat16), d, rotated, inter, eps)


def test_keys_next_to_the_middle_of_two_bf16_values():
    """A key's two roundings, 64 bits to fp32 and from there to bf16: what fp32
    rounds to the middle of two bf16 values goes to the even one.  k times the
    factor is m (1 - 2^-13) (1 + 2^-13) = m (1 - 2^-26), less than an eighth of
    fp32's step below the middle m."""
    D = _D()
    d, rows = 128, 127
    m = torch.arange(128, 255).double() + 0.5
    k = (m * (1 - 2.0 ** -13)).float()
    assert (k.double() == m * (1 - 2.0 ** -13)).all()
    k = k[:, None, None].expand(rows, 1, d).contiguous().to(DEV)
    store = _store(D, [rows], 1, d, D.DOPR_STORE_BF16)
    D.dopr_store_put_rotary(
        store, 0, torch.zeros(1, dtype=torch.int32, device=DEV),
        torch.tensor([0, rows], device=DEV), k, k,
        torch.zeros(d // 2, device=DEV), attention_factor=1 + 2.0 ** -13)
    got, _ = _gather(D, store, 0, [0], _cu([rows]), 1, d)
    even = 2 * ((m + 0.5) / 2).floor()
    assert (got[:, 0].double() == even[:, None]).all()
