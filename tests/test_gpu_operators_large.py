"""The operators at sizes that one launch does not take (GPU): more rows,
tokens or columns than 2^32 threads allow, of a few bytes each."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    gc.collect()
    torch.cuda.empty_cache()


def _D():
    import paper_2609_03311_amd as D
    return D


ROWS = (1 << 26) + 5


def test_rows_and_norms():
    """Every row is 8 values of +-2^e: its 8-bit form is +-127, its scale
    2^e / 127, its norm (without an epsilon) +-1, all without rounding but
    the scale's."""
    D = _D()
    e = (torch.arange(ROWS, device=DEV) % 15 - 7).to(torch.float32)
    value = torch.exp2(e)
    x = value.to(torch.float16)[:, None].repeat(1, 8)
    x[:, 3] *= -1
    sign = torch.ones(8, device=DEV)
    sign[3] = -1
    q = torch.zeros(ROWS, 8, dtype=torch.int8, device=DEV)
    s = torch.zeros(ROWS, device=DEV)
    D.dopr_quantize_rows(x, q, s)
    assert (q == (127 * sign).to(torch.int8)).all()
    assert torch.equal(s, value / 127)
    z = torch.zeros_like(x)
    q.zero_()
    s.zero_()
    D.dopr_norm_residual(x, pre_norm_w=torch.ones_like(x[0]), z=z, q=q,
                         q_scale=s, rms_eps=0.0)
    assert (z == sign.to(torch.float16)).all()
    assert (q == (127 * sign).to(torch.int8)).all()
    assert (s == torch.tensor(1.0) / 127).all()


def test_tokens():
    """Positions of a quarter turn: (a, b) to (b, -a) and so on."""
    D = _D()
    x = torch.arange(ROWS, device=DEV, dtype=torch.float32)[:, None]
    x = torch.cat((x % 251, x % 127), 1).to(torch.bfloat16)[:, None, :]
    pos = (torch.arange(ROWS, device=DEV) % 4).to(torch.int32)
    out = torch.zeros_like(x)
    quarter = torch.tensor([torch.pi / 2], device=DEV)
    D.dopr_rotary(x, None, pos, quarter, out, None)
    cos = torch.tensor([1.0, 0.0, -1.0, 0.0], device=DEV)[pos.long()]
    sin = torch.tensor([0.0, 1.0, 0.0, -1.0], device=DEV)[pos.long()]
    a, b = x[:, 0, 0].float(), x[:, 0, 1].float()
    # the quarter is off by 2^-24 of itself, three of them by under 2^-21
    for got, want in ((out[:, 0, 0], a * cos - b * sin),
                      (out[:, 0, 1], b * cos + a * sin)):
        assert ((got.float() - want).abs() <= 2.0 ** -21 * 256).all()


def _codes(n, step):
    """n int8 values and n scales, powers of two."""
    i = torch.arange(n, device=DEV)
    return ((i * step) % 255 - 127).to(torch.int8), torch.exp2(
        (i % 5 - 2).to(torch.float32))


def test_columns_of_few_rows():
    D = _D()
    n = (1 << 27) + 37
    w, ws = _codes(n, 7)
    x, xs = _codes(3, 31)
    y = torch.zeros(3, n, dtype=torch.float32, device=DEV)
    D.dopr_quant_matmul(x[:, None], xs, w[:, None], ws, y)
    for m in range(3):
        assert torch.equal(y[m], w.float() * float(x[m]) * float(xs[m]) * ws)


@pytest.mark.parametrize("m,laid_out", [((1 << 29) + 77, False),
                                        ((1 << 28) + 77, True)])
def test_rows_of_one_column(m, laid_out):
    """As they lie, and laid out again in a workspace of 34 GB."""
    D = _D()
    x, xs = _codes(m, 7)
    w, ws = _codes(1, 31)
    w[:] = -77
    y = torch.zeros(m, 1, dtype=torch.float32, device=DEV)
    wsp = torch.empty((m + 1) * 128, dtype=torch.uint8,
                      device=DEV) if laid_out else None
    D.dopr_quant_matmul(x[:, None], xs, w[:, None], ws, y, workspace=wsp)
    assert torch.equal(y[:, 0], x.float() * -77.0 * xs * float(ws[0]))
