"""The no-alloc call over a 4-bit store past its scratch: the block kernels in
place of the ones that need no plan."""
import pytest

from test_gpu_fp4_rows import Rows, _same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv,pairs,norm", [
    (128, 2, 2, 700, True), (64, 4, 4, 1000, False)])
def test_calls_past_the_scratch(d, hq, hkv, pairs, norm):
    import paper_2609_03311_amd as D
    tokens = [100 - p % 7 for p in range(pairs)]
    r = Rows([40, 0, 77, -1, 33], [p % 6 for p in range(pairs)], tokens, hq,
             hkv, d, norm=norm, seed=d, freq=norm)
    # k^ and the rotations alone are more than the scratch holds
    assert (2 * hkv * d + 4 * d) * r.total > D.DOPR_NOALLOC_SCRATCH_BYTES
    got = r.call(noalloc=True)
    _same(got, r.call(variant=6))
    # (every unit one wave's: the automatic choice's bits)
    _same(got, r.call())
    assert D.dopr_check_status(r.store) == D.DOPR_ERR_DOC_RANGE
    less, _ = r.call(noalloc=True, lse=False)
    _same((less,), got[:1])
