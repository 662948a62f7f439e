"""Every way an int8 product runs (GPU), compared bit for bit.

The integer sum is exact, the scales here are powers of two, and what follows is
one fp32 addition each for bias and residual and the rounding to the output's
type: the same steps in torch give the same bits.  Sums stay below 2^28, so the
scaled ones neither overflow nor lose bits to subnormals."""
import pytest
import torch

from product_sizes import SIZES
from test_gpu_operators import DEV, TYPES, Guarded, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", SIZES)
def test_product_bit_for_bit(m, n, k):
    import paper_2609_03311_amd as D
    g = gen(m + n + k)

    def codes(rows):
        to = Guarded(rows, k, torch.int8, gap=-k % 16)
        return to.set(torch.randint(-128, 128, (rows, k), generator=g,
                                    device=DEV, dtype=torch.int8))

    def scales(count, low):
        return torch.exp2(torch.randint(low, low + 4, (count,), generator=g,
                                        device=DEV).float())

    x, w = codes(m), codes(n)
    assert x.data_ptr() % 16 == w.data_ptr() % 16 == 0
    xs, ws = scales(m, -9), scales(n, -11)
    want = (x.double() @ w.double().t()).float()
    want = want * xs[:, None] * ws[None, :]
    for dtype in TYPES:
        # rows of y on their own stride and off it
        y = Guarded(m, n, dtype)
        D.dopr_quant_matmul(x, xs, w, ws, y.view)
        assert torch.equal(y.view, want.to(dtype)), dtype
        y.check()
        y = Guarded(m, n, dtype, gap=3, offset=1)
        bias = randn(g, n, dtype=dtype)
        r = y.set(randn(g, m, n, dtype=dtype))
        ref = (want + bias.float() + r.float()).to(dtype)
        D.dopr_quant_matmul(x, xs, w, ws, r, bias=bias, residual=r)
        assert torch.equal(y.view, ref), dtype
        y.check()
