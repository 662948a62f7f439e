"""Attention over a 4-bit store past 32 bits whose answer hangs on single slots
there (as in test_gpu_fp4_marks.py: no rotation, a scale of ln 2): a document of
more than 4 GB and one behind it, marked slots at both ends and on both sides of
the 2^31st and the 2^32nd byte.

Values are 1 in one dim a region (a 128th of a document), 6 in one more at a
marked slot.  With q = 0 the normaliser is the number of keys, below 2^24 and
exact, and each dim the share of its region.  With two marked keys at logits x
and y (log2 units) over the others' 0 a row is
(sum of v + (2^x - 1) v_a + (2^y - 1) v_b) / (n + 2^x + 2^y - 2).  A wave adds
its chunks in turn, in fp32, under 2^12 of them: 2^-12 of the marked terms, and
the others, n 2^-x of them, may be lost beside them; the output's rounding is
2^-8."""
import gc
import math

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


def test_slots_past_4_gb():
    import paper_2609_03311_amd as D
    hkv, rep, d, lens = 8, 2, 128, [4_200_000, 3000]
    hq = hkv * rep
    at = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    rows = int(at[-1])
    k, v = (torch.zeros((rows, hkv, d), dtype=torch.bfloat16, device=DEV)
            for _ in range(2))
    chunk_bytes = 34 * d
    head_bytes = -(-lens[0] // 32) * chunk_bytes
    marks = [[0, 31, 32, lens[0] - 1, lens[0] - 32], [0, 1500, lens[1] - 1]]
    for edge in (1 << 31, 1 << 32):
        c = edge % head_bytes // chunk_bytes
        marks[0] += [32 * c - 1, 32 * c, 32 * c + 31, 32 * c + 32]
    heads = torch.arange(hkv, device=DEV)
    for doc, n in enumerate(lens):
        first = int(at[doc])
        s = torch.arange(n, device=DEV)
        region = s // 32 * d // (-(-n // 32))
        for g in range(hkv):
            v[first + s, g, (region + 5 * g) % d] = 1.0
        for i, slot in enumerate(marks[doc]):
            k[first + slot, :, i] = 6.0
            v[first + slot, heads, (64 + 7 * i + 3 * heads) % d] = 6.0
        del s, region
    store = D.dopr_store_create(1, hkv, d, np.asarray(lens, np.int32),
                                format=D.DOPR_STORE_FP4)
    assert hkv * head_bytes > 1 << 32
    D.dopr_store_put(store, 0,
                     torch.tensor([0, 1], dtype=torch.int32, device=DEV),
                     torch.from_numpy(at).to(DEV), k, v)
    sums = [torch.stack([v[a:b, g].sum(0, dtype=torch.float64)
                         for g in range(hkv)]).cpu()
            for a, b in zip(at[:-1], at[1:])]
    marked = [v[torch.tensor(m, device=DEV) + int(a)].double().cpu()
              for m, a in zip(marks, at)]       # [mark, head, dim]
    del k, v
    gen = torch.Generator().manual_seed(1)
    for tokens, docs in (([1, 1], [0, 1]), ([3, 1], [1, 0]), ([1, 3], [1, 0])):
        total = sum(tokens)
        tcu = np.concatenate([[0], np.cumsum(tokens)]).astype(np.int32)
        shape = dict(max_tokens=max(tokens), total_tokens=total)
        ws = torch.full((max(256, D.dopr_prefix_attn_workspace(
            store, n_pairs=2, n_q_heads=hq, **shape)),), 255,
            dtype=torch.uint8, device=DEV)
        own_v = torch.randint(-4, 5, (total, hkv, d), generator=gen).double()

        def call(q):
            out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16,
                             device=DEV)
            lse = torch.full((total, hq), float("nan"), device=DEV)
            D.dopr_prefix_attn(
                store, 0, torch.tensor(docs, dtype=torch.int32, device=DEV),
                torch.from_numpy(tcu).to(DEV), q.to(DEV, torch.bfloat16),
                torch.zeros((total, hkv, d), dtype=torch.bfloat16,
                            device=DEV), own_v.to(DEV, torch.bfloat16), None,
                None, out, ws, lse=lse, softmax_scale=math.log(2.0),
                rope_inv_freq=torch.zeros(d // 2, device=DEV), **shape)
            return out.cpu().double(), lse.cpu().double()

        places = [(p, int(tcu[p]) + j, j) for p in range(2)
                  for j in range(tokens[p])]
        out, lse = call(torch.zeros(total, hq, d))
        for p, t, j in places:
            n = lens[docs[p]] + j + 1
            own = own_v[t - j:t + 1].sum(0)
            want = (sums[docs[p]] + own).repeat_interleave(rep, 0) / n
            # (own values, of either sign, next to the sum of the prefix's)
            slack = 2.0 ** -20 * (want.abs() + 12 * (j + 1) / n)
            assert ((out[t] - want).abs() <= 2.0 ** -8 * want.abs()
                    + slack).all(), (docs, p, j)
            assert ((lse[t] - math.log(n)).abs()
                    <= 2.0 ** -21 * math.log(n)).all(), (docs, p, j)
        most = max(len(m) for m in marks)
        for turn in range(most):
            q = torch.zeros(total, hq, d)
            plan = []
            for p, t, j in places:
                m = len(marks[docs[p]])
                for h in range(hq):
                    a, b = (turn + h) % m, (turn + 2 * h + 1) % m
                    b = b if b != a else (b + 1) % m
                    low = 6 - 0.5 * (h % 4)
                    q[t, h, a], q[t, h, b] = 6.0, low
                    plan.append((p, t, j, h, a, b, 36.0, 6 * low))
            out, lse = call(q)
            for p, t, j, h, a, b, x, y in plan:
                g, doc = h // rep, docs[p]
                n = lens[doc] + j + 1
                fa, fb = 2.0 ** x - 1, 2.0 ** y - 1
                va, vb = marked[doc][a, g], marked[doc][b, g]
                own = own_v[t - j:t + 1, g]
                total_w = n + fa + fb
                want = (sums[doc][g] + own.sum(0) + fa * va + fb * vb) / total_w
                slack = (sums[doc][g] + own.abs().sum(0) + 2.0 ** -12
                         * (fa * va + fb * vb)) / total_w
                off = (out[t, h] - want).abs()
                assert (off <= 2.0 ** -8 * want.abs() + slack).all(), (
                    docs, p, j, h, marks[doc][a], marks[doc][b], off.max())
                log = math.log(total_w)
                assert abs(lse[t, h] - log) <= 2.0 ** -20 * log + 2.0 ** -12, (
                    docs, p, j, h, float(lse[t, h]), log)
    assert D.dopr_check_status(store) == D.DOPR_OK
