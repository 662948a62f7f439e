"""States put into a 4-bit store (and a bf16 one) by a captured graph, replayed
with other states, positions and documents and eager work between."""
import numpy as np
import pytest
import torch

from test_gpu_fp4_store import _cu, _gen, _same

pytestmark = pytest.mark.gpu

DEV = "cuda"


# ten documents' chunks in blocks of their own, whose bounds a launch in front
# clears; and more documents than blocks are shared for
@pytest.mark.parametrize("lens", [[40, 300, 0, 33] * 2, [7] * 5000])
@pytest.mark.parametrize("fmt", [0, 1])
def test_put_rotary_replayed(lens, fmt):
    import paper_2609_03311_amd as D
    hkv, d = 2, 64
    cu = _cu(lens)
    rows, n = int(cu[-1]), len(lens)
    ids = torch.arange(n, dtype=torch.int32, device=DEV)
    at = torch.from_numpy(cu).to(DEV)
    k, v = (torch.zeros((rows, hkv, d), dtype=torch.float16, device=DEV)
            for _ in range(2))
    pos = torch.zeros(rows, dtype=torch.int32, device=DEV)
    gain = torch.ones(d, dtype=torch.float16, device=DEV)
    freq = (1e4 ** (-torch.arange(0, d, 2) / d)).to(DEV)
    stores = [D.dopr_store_create(1, hkv, d, np.asarray(lens, np.int32),
                                  format=fmt) for _ in range(2)]
    read = [[torch.zeros((rows, hkv, d), dtype=torch.bfloat16, device=DEV)
             for _ in range(2)] for _ in stores]

    def fill(store, out):
        s = torch.cuda.current_stream()
        D.dopr_store_put_rotary(store, 0, ids, at, k, v, freq, positions=pos,
                                k_norm_w=gain, stream=s)
        D.dopr_gather_prefix(store, 0, ids, at, *out, stream=s)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        fill(stores[0], read[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        fill(stores[0], read[0])
    for i in range(4):
        gen = _gen(i)
        for x in (k, v):
            x.copy_(torch.randn(x.shape, generator=gen) * 2.0 ** -i)
        pos.copy_(torch.randint(0, 9000, (rows,), generator=gen))
        gain.copy_(1 + 0.1 * torch.randn(d, generator=gen))
        for x in read[0]:
            x.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in read[0]]
        fill(stores[1], read[1])
        torch.cuda.synchronize()
        for a, b in zip(got, read[1]):
            assert _same(a, b), i
        # (the bounds of the keys are those of the states there now)
        one = [torch.randn((n, h, d), generator=gen).to(DEV, torch.bfloat16)
               for h in (4, hkv, hkv)]
        outs = []
        for st in stores:
            ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
            out = torch.zeros_like(one[0])
            D.dopr_prefix_attn(
                st, 0, ids, torch.arange(n + 1, dtype=torch.int32,
                                         device=DEV), *one, None, None, out,
                ws, max_tokens=1, total_tokens=n)
            outs.append(out)
        assert _same(*outs), i
    for st in stores:
        assert D.dopr_check_status(st) == D.DOPR_OK
