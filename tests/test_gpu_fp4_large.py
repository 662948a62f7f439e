"""A 4-bit store past 32 bits: offsets of documents, heads and chunks."""
import gc

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    gc.collect()
    torch.cuda.empty_cache()


def test_a_document_of_more_than_4_gb():
    """Values that 4 bits hold exactly, so what is read back is what was put;
    attention of one token and of three over the first and last kv heads,
    against 64 bits.  Beside the roundings that the shorter tests count (q^ and
    k^ 2^-8 of each product, a weight 2^-8), a wave adds its chunks' sums in
    fp32: under 2^12 terms, 2^-12."""
    import paper_2609_03311_amd as D
    hkv, hq, d, lens = 8, 16, 128, [4_200_000, 3000]
    at = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    rows = int(at[-1])
    gen = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.empty((rows, hkv, d), dtype=torch.bfloat16, device=DEV)
            .random_(-4, 5, generator=gen) for _ in range(2))
    # each block's largest is 6: a key's of every (64-dim part, half) and a
    # value's of every 32 slots, counted from the document's first
    k.view(rows, hkv, 2, 4, 2, 8)[:, :, :, 0, :, 0] = 6.0
    v[0:lens[0]:32] = -6.0
    v[lens[0]::32] = -6.0
    store = D.dopr_store_create(1, hkv, d, np.asarray(lens, np.int32),
                                format=D.DOPR_STORE_FP4)
    assert store.pool.numel() > 1 << 32
    ids = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    cu = torch.from_numpy(at).to(DEV)
    D.dopr_store_put(store, 0, ids, cu, k, v)
    for x in (k, v):
        pair = [torch.full_like(x, 9.0), torch.empty_like(x)]
        if x is v:
            pair.reverse()
        D.dopr_gather_prefix(store, 0, ids, cu, *pair)
        assert torch.equal(pair[0] if x is k else pair[1], x)
        del pair
    freq = (1e6 ** (-torch.arange(0, d, 2).double() / d)).float()
    for tokens, docs in (([1, 1], [0, 1]), ([3, 1], [1, 0]), ([1, 3], [1, 0])):
        total = sum(tokens)
        q, own_k, own_v = (
            (s * torch.randn((total, h, d), generator=gen, device=DEV))
            .to(torch.bfloat16) for h, s in ((hq, 0.2), (hkv, 1.0),
                                             (hkv, 1.0)))
        tcu = np.concatenate([[0], np.cumsum(tokens)]).astype(np.int32)
        shape = dict(max_tokens=max(tokens), total_tokens=total)
        ws = torch.empty(max(256, D.dopr_prefix_attn_workspace(
            store, n_pairs=2, n_q_heads=hq, **shape)), dtype=torch.uint8,
            device=DEV)
        out = torch.zeros_like(q)
        D.dopr_prefix_attn(store, 0, torch.tensor(docs, dtype=torch.int32,
                                                  device=DEV),
                           torch.from_numpy(tcu).to(DEV), q, own_k, own_v,
                           None, None, out, ws,
                           rope_inv_freq=freq.to(DEV), **shape)
        for p in range(2):
            a, b = int(tcu[p]), int(tcu[p + 1])
            L, first = lens[docs[p]], int(at[docs[p]])
            t = (L + torch.arange(b - a, device=DEV).double())[:, None, None]
            t = t * freq.to(DEV).double()

            def turned(x):
                x = x[a:b].double()
                one, two = x[..., :d // 2], x[..., d // 2:]
                c, s = t.cos(), t.sin()
                return torch.cat((one * c - two * s, two * c + one * s), -1)

            qt, kt = turned(q), turned(own_k)
            for g in (0, hkv - 1):
                keys = torch.cat((k[first:first + L, g].double(), kt[:, g]))
                vals = torch.cat((v[first:first + L, g].double(),
                                  own_v[a:b, g].double()))
                for j in range(b - a):
                    n = L + j + 1
                    x = qt[j, 2 * g:2 * g + 2] @ keys[:n].T * d ** -0.5
                    w = torch.softmax(x, -1)
                    want = w @ vals[:n]
                    m = w @ vals[:n].abs()
                    size = (qt[j, 2 * g:2 * g + 2].abs() @ keys[:n].abs().T
                            * d ** -0.5).amax(-1, keepdim=True)
                    e = 2.0 ** -8 + 2.0 ** -12 + 2.0 ** -6.9 * size
                    got = out[a + j, 2 * g:2 * g + 2].double()
                    assert ((got - want).abs() <= 2.02 * e * m
                            + 2.0 ** -8 * want.abs()).all(), (docs, p, g, j)
    assert D.dopr_check_status(store) == D.DOPR_OK
