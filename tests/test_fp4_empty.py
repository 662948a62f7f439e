"""Documents without slots on their way into a store: no rows, so no memory (a
tensor of no elements has no address)."""
import pytest

from store_calls import store_calls
from test_fp4_abi import INVALID, _put


@pytest.mark.parametrize("fmt", [0, 1])
def test_no_rows_need_no_memory(fmt):
    got = store_calls((2, 2, 128, [0, 0, 5], fmt), [
        _put(rows=0, k=None, v=None), _put(rows=1, k=None),
        _put(rows=1, v=None), _put(rows=0, k=None, v=None, doc_ids=None)])
    assert got[0]["status"] == 0, got[0]["error"]
    assert got[0]["launches"]
    for g in got[1:]:
        assert g["status"] == INVALID and "NULL" in g["error"]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("lens", [[0, 0], [0, 40, 0]])
def test_documents_without_slots(fmt, lens):
    """Put alone, next to one that a call without rows may not read."""
    import numpy as np
    import torch
    import paper_2609_03311_amd as D
    store = D.dopr_store_create(1, 2, 64, np.asarray(lens, np.int32),
                                format=fmt)
    n = len(lens)
    none = torch.empty(0, 2, 64, device="cuda")
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    cu = torch.tensor([0] + list(np.cumsum(lens)), device="cuda")
    D.dopr_store_put_rotary(
        store, 0, ids, cu, none, none, torch.ones(32, device="cuda"),
        positions=torch.empty(0, dtype=torch.int32, device="cuda"))
    assert D.dopr_check_status(store) == (
        D.DOPR_ERR_DOC_RANGE if 40 in lens else D.DOPR_OK)
