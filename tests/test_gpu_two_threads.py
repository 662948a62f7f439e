"""Two Python threads in the compiled calls at once, each with its own stream,
workspace and outputs: the results of calls made in turn."""
import threading

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"


class Work:
    def __init__(self, seed):
        import paper_2609_03311_amd as D
        self.D, hkv, d = D, 2, 128
        gen = torch.Generator().manual_seed(seed)

        def randn(*shape, dtype=torch.bfloat16):
            return torch.randn(shape, generator=gen).to(DEV, dtype)

        lens = np.array([70, 300, 33], np.int32)
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        self.ids = torch.arange(3, dtype=torch.int32, device=DEV)
        self.at = torch.from_numpy(cu).to(DEV)
        self.k, self.v = randn(int(cu[-1]), hkv, d), randn(int(cu[-1]), hkv, d)
        self.freq = (1e6 ** (-torch.arange(0, d, 2) / d)).to(DEV)
        self.stores = [D.dopr_store_create(1, hkv, d, lens, format=f)
                       for f in (0, 1)]
        self.tokens = [5, 40, 17]
        self.tcu = torch.tensor([0, 5, 45, 62], dtype=torch.int32, device=DEV)
        self.own = [randn(62, h, d) for h in (4, hkv, hkv)]
        self.x = randn(100, 256)
        self.w = torch.randint(-127, 128, (64, 256), generator=gen).to(
            DEV, torch.int8)
        self.w_scale = torch.rand(64, generator=gen).to(DEV)
        self.ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
        self.stream = torch.cuda.Stream()

    def run(self):
        """Every compiled call, in the order of their streams; the outputs."""
        D, s, out = self.D, self.stream, []
        with torch.cuda.stream(s):
            for st in self.stores:
                D.dopr_store_put_rotary(st, 0, self.ids, self.at, self.k,
                                        self.v, self.freq, stream=s)
                read = [torch.empty_like(self.k) for _ in range(2)]
                D.dopr_gather_prefix(st, 0, self.ids, self.at, *read,
                                     stream=s)
                o = torch.empty_like(self.own[0])
                D.dopr_prefix_attn(st, 0, self.ids, self.tcu, *self.own, None,
                                   None, o, self.ws, max_tokens=40,
                                   total_tokens=62, rope_inv_freq=self.freq,
                                   stream=s)
                out += read + [o]
            q = torch.empty(100, 256, dtype=torch.int8, device=DEV)
            scale = torch.empty(100, device=DEV)
            D.dopr_quantize_rows(self.x, q, scale, stream=s)
            y = torch.empty(100, 64, dtype=torch.bfloat16, device=DEV)
            D.dopr_quant_matmul(q, scale, self.w, self.w_scale, y,
                                workspace=self.ws, stream=s)
            z = torch.empty_like(self.x)
            D.dopr_norm_residual(self.x, pre_norm_w=self.x[0].clone(), z=z,
                                 stream=s)
            r = torch.empty_like(self.k)
            D.dopr_rotary(None, self.k, torch.arange(
                self.k.shape[0], dtype=torch.int32, device=DEV), self.freq,
                None, r, stream=s)
        return out + [q, scale, y, z, r]


def test_two_threads_at_once():
    work = [Work(1), Work(2)]
    torch.cuda.synchronize()
    want = []
    for w in work:
        want.append(w.run())
        torch.cuda.synchronize()
    got, errors = [[], []], []

    def loop(i):
        try:
            for _ in range(20):
                got[i].append(work[i].run())
        except BaseException as e:  # (named by the test)
            errors.append(e)

    threads = [threading.Thread(target=loop, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for i in range(2):
        assert len(got[i]) == 20
        for run in got[i]:
            for a, b in zip(run, want[i]):
                assert torch.equal(a, b)
