"""Prefix attention over a 4-bit store without a plan (the automatic way of
pairs of several tokens): rows that one wave forms, bit for bit the planned
kernels'; rows that several share, against the definition in 64 bits.

What the kernels round against that definition: q^ and k^ once to bf16 (2^-8 of
each product q_d k_d), each softmax weight once to bf16 in the weighted sum and
the normaliser alike, the output once to bf16; the rest is fp32.  With A = sum
of weight * |value| and S = the largest sum of |q_d k_d| (natural-log units) of
a row, weights off by e = 2^-8 + 2^-6.9 S (two roundings of 2^-8 and their
product, fp32's beside them) move the row by at most 2 e A, the rounding by
2^-8 of the row, and the log-sum-exp by e."""
import numpy as np
import pytest
import torch

import fp4_refs

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _D():
    import paper_2609_03311_amd as D
    return D


class Rows:
    def __init__(self, lens, docs, tokens, hq, hkv, d, *, norm=True, seed=0,
                 scale=1.0, gain=1.0, freq=True, layers=1, layer=0):
        D = _D()
        gen = torch.Generator().manual_seed(seed)

        def randn(*shape):
            return torch.randn(shape, generator=gen)

        self.lens, self.docs, self.layer = lens, docs, layer
        res = [i for i, n in enumerate(lens) if n >= 0]
        at = np.concatenate([[0], np.cumsum([lens[i] for i in res])])
        k = (randn(int(at[-1]), hkv, d) * scale).to(torch.bfloat16)
        v = randn(int(at[-1]), hkv, d).to(torch.bfloat16)
        self.hk, self.hv = fp4_refs.held(k, v, at)
        self.rows = {i: slice(int(a), int(b))
                     for i, a, b in zip(res, at[:-1], at[1:])}
        self.store = D.dopr_store_create(layers, hkv, d,
                                         np.asarray(lens, np.int32),
                                         format=D.DOPR_STORE_FP4)
        D.dopr_store_put(self.store, layer,
                         torch.tensor(res, dtype=torch.int32, device=DEV),
                         torch.from_numpy(at).to(DEV), k.to(DEV), v.to(DEV))
        self.n, self.hq, self.hkv, self.d = len(docs), hq, hkv, d
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(tokens)]),
                               dtype=torch.int32)
        self.total, self.most = int(self.cu[-1]), max(tokens)
        self.q = randn(self.total, hq, d).to(torch.bfloat16)
        self.k = (randn(self.total, hkv, d)
                  * (scale if not norm else 1.0)).to(torch.bfloat16)
        self.v = randn(self.total, hkv, d).to(torch.bfloat16)
        self.qw = self.kw = None
        if norm:
            self.qw, self.kw = ((gain * (1 + 0.1 * randn(d))).to(
                torch.bfloat16) for _ in range(2))
        self.freq = 1e6 ** (-torch.arange(0, d, 2).double() / d)
        self.given = self.freq.float().to(DEV) if freq else None
        if freq:
            self.freq = self.freq.float().double()

    def inputs(self, cu=None):
        return [None if x is None else x.to(DEV) for x in
                (torch.tensor(self.docs, dtype=torch.int32),
                 self.cu if cu is None else cu, self.q, self.k, self.v,
                 self.qw, self.kw)]

    def workspace(self, variant=0, most=None):
        D = _D()
        need = D.dopr_prefix_attn_workspace(
            self.store, n_pairs=self.n, n_q_heads=self.hq,
            max_tokens=most or self.most, total_tokens=self.total,
            kernel_variant=variant)
        # (filled with what no call may take for its own)
        return torch.full((max(need, 256),), 255, dtype=torch.uint8,
                          device=DEV)

    def call(self, *, lse=True, variant=0, noalloc=False, cu=None, out=None,
             most=None, inputs=None, workspace=None, stream=None):
        D = _D()
        if out is None:
            out = torch.full((self.total, self.hq, self.d), 3.0,
                             dtype=torch.bfloat16, device=DEV)
        lse = (torch.full((self.total, self.hq), 3.0, device=DEV) if lse
               else None)
        inputs = inputs or self.inputs(cu)
        kw = dict(max_tokens=most or self.most, lse=lse,
                  total_tokens=self.total, rope_inv_freq=self.given,
                  kernel_variant=variant, stream=stream)
        if noalloc:
            D.dopr_prefix_attn_noalloc(self.store, self.layer, *inputs, out,
                                       **kw)
        else:
            if workspace is None:
                workspace = self.workspace(variant, most)
            D.dopr_prefix_attn(self.store, self.layer, *inputs, out,
                               workspace, **kw)
        return out, lse

    def check(self, out, lse):
        out, lse = out.cpu().double(), lse.cpu().double()
        scale, rep = self.d ** -0.5, self.hq // self.hkv
        for p in range(self.n):
            a, b = int(self.cu[p]), int(self.cu[p + 1])
            doc, n = self.docs[p], b - a
            if not 0 <= doc < len(self.lens) or self.lens[doc] < 0:
                assert (out[a:b] == 0).all()
                assert (lse[a:b] == -float("inf")).all()
                continue
            L = self.lens[doc]
            t = (L + torch.arange(n)).double()[:, None, None]

            def formed(x, w):
                x = x[a:b].double()
                if w is not None:
                    x = x / torch.sqrt(x.square().mean(-1, keepdim=True)
                                       + 1e-6) * w.double()
                u, v = x[..., :self.d // 2], x[..., self.d // 2:]
                c, s = (t * self.freq).cos(), (t * self.freq).sin()
                return torch.cat((u * c - v * s, v * c + u * s), -1)

            q, k = formed(self.q, self.qw), formed(self.k, self.kw)
            keys = torch.cat((self.hk[self.rows[doc]].double(), k))
            vals = torch.cat((self.hv[self.rows[doc]].double(),
                              self.v[a:b].double()))
            hide = torch.full((n, n), -float("inf")).double().triu(1)
            hide = torch.cat((torch.zeros((n, L)).double(), hide), 1)
            for h in range(self.hq):
                g = h // rep
                x = q[:, h] @ keys[:, g].T * scale + hide
                w = torch.softmax(x, -1)
                o, m = w @ vals[:, g], w @ vals[:, g].abs()
                size = (q[:, h].abs() @ keys[:, g].abs().T * scale)
                size = torch.where(hide == 0, size, 0.0).amax(-1)
                e = (2.0 ** -8 + 2.0 ** -6.9 * size)[:, None]
                off = (out[a:b, h] - o).abs()
                assert (off <= 2.02 * e * m + 2.0 ** -8 * o.abs()
                        + 1e-30).all(), (p, h, off.max())
                want = torch.logsumexp(x, -1)
                assert ((lse[a:b, h] - want).abs() <= 1.01 * e[:, 0]
                        + 2.0 ** -20 * want.abs()).all(), (p, h)


def _same(a, b):
    for x, y in zip(a, b):
        x, y = x.cpu().contiguous(), y.cpu().contiguous()
        kind = torch.int16 if x.dtype == torch.bfloat16 else torch.int32
        assert torch.equal(x.view(kind), y.view(kind))


FEW = [
    # lens, docs, tokens, q heads, kv heads: units that waves share
    ([5], [0], [2], 4, 4),
    ([0, 33], [0, 1, 1], [3, 40, 70], 8, 2),
    ([256], [0], [129], 32, 8),
    ([90, -1, 300], [0, 2, 1, 9, 0], [17, 31, 5, 9, 66], 15, 3),
    ([3000], [0, 0], [33, 1], 8, 1),
    ([40], [0], [300], 3, 1),
    ([10, 70], [1, 0], [8, 200], 40, 1),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("shape", range(len(FEW)))
def test_few_rows(d, norm, shape):
    r = Rows(*FEW[shape], d, norm=norm, seed=shape, freq=norm)
    got = r.call()
    r.check(*got)
    bare, none = r.call(lse=False)
    assert none is None and torch.equal(bare, got[0])
    _same(r.call(noalloc=True), got)
    # a loose bound on the tokens of a pair
    _same(r.call(most=5000), got) if r.total > 5000 else r.check(
        *r.call(most=5000))


@pytest.mark.parametrize("lens,docs,tokens,hq,hkv", [
    ([20001], [0], [7], 4, 1), ([513, 6000], [1, 0, 1], [3, 2, 5], 8, 2)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("norm", [True, False])
def test_long_prefixes_are_split(lens, docs, tokens, hq, hkv, d, norm):
    r = Rows(lens, docs, tokens, hq, hkv, d, norm=norm, seed=5)
    r.check(*r.call())


@pytest.mark.parametrize("scale,gain,norm", [
    (40.0, 1.0, True), (1.0, 8.0, True), (40.0, 1.0, False),
    (2.0 ** -40, 1.0, True)])
@pytest.mark.parametrize("lens", [[40, 300, 0], [4000, 10, 1000]])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_of_any_size(scale, gain, norm, lens, d):
    r = Rows(lens, [0, 1, 2, 0], [5, 40, 33, 2], 8, 2, d, norm=norm, seed=6,
             scale=scale, gain=gain)
    r.check(*r.call())


def _many(d, norm, n_rep, seed=1, scale=1.0):
    """Enough rows that a wave forms each alone."""
    rng = np.random.default_rng(seed)
    lens = [int(x) for x in rng.integers(0, 200, 60)] + [-1]
    docs = [int(x) for x in rng.integers(0, 62, 300)]
    tokens = [int(x) for x in rng.integers(1, 90, 300)]
    return Rows(lens, docs, tokens, 4 * n_rep, 4, d, norm=norm, seed=seed,
                scale=scale)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("n_rep", [1, 2, 3, 4, 8])
def test_many_rows_are_the_planned_kernels(d, norm, n_rep):
    r = _many(d, norm, n_rep)
    want = r.call(variant=8)
    _same(r.call(), want)
    _same(r.call(most=r.total), want)
    assert _D().dopr_check_status(r.store) == _D().DOPR_ERR_DOC_RANGE


@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_out_of_range(d):
    """Without QK-norm, rows whose normaliser leaves the safe range are run
    again with the exact maximum."""
    r = _many(d, False, 4, seed=2, scale=30.0)
    out, lse = r.call()
    exact = r.call(variant=4)
    assert torch.isfinite(lse[lse != -float("inf")]).all()
    assert lse.max() > 100
    # (both round q^, k^ and the weights alike; sums in another order)
    assert (lse - exact[1])[lse != -float("inf")].abs().max() < 1e-2
    assert (out.float() - exact[0].float()).abs().max() < 0.05


def test_malformed_token_ranges():
    D = _D()
    r = Rows([40, 33], [0, 1, 0], [3, 4, 5], 4, 2, 64, seed=9)
    want, _ = r.call()
    out = torch.full_like(want, 3.0)
    r.call(cu=torch.tensor([0, 3, 3, 12], dtype=torch.int32), out=out, most=9)
    assert D.dopr_check_status(r.store) == D.DOPR_ERR_SEQLEN
    assert torch.equal(out[:3], want[:3])
    for bad in ([1, 3, 7, 12], [0, 3, 7, 13], [0, 7, 3, 12], [0, 3, 7, 11],
                [-4, 3, 7, 12], [0, 12, 12, 12]):
        r.call(cu=torch.tensor(bad, dtype=torch.int32))
        assert D.dopr_check_status(r.store) == D.DOPR_ERR_SEQLEN


@pytest.mark.parametrize("shape", [2, 4, None])
def test_graph_replays(shape):
    """A captured call, replayed with other inputs and eager work between."""
    D = _D()
    r = (Rows(*FEW[shape], 128, seed=3) if shape is not None
         else _many(64, True, 2))
    bufs, ws = r.inputs(), r.workspace()
    out = torch.zeros((r.total, r.hq, r.d), dtype=torch.bfloat16, device=DEV)
    s = torch.cuda.Stream()

    def call():
        D.dopr_prefix_attn(r.store, 0, *bufs, out, ws, max_tokens=r.most,
                           total_tokens=r.total, rope_inv_freq=r.given,
                           stream=torch.cuda.current_stream())

    with torch.cuda.stream(s):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    for i in range(4):
        gen = torch.Generator().manual_seed(i)
        r.q = torch.randn(r.q.shape, generator=gen).to(torch.bfloat16)
        r.k = torch.randn(r.k.shape, generator=gen).to(torch.bfloat16)
        bufs[2].copy_(r.q)
        bufs[3].copy_(r.k)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want, _ = r.call()
        assert torch.equal(got, want), i


def test_layers():
    r = Rows([90, 20], [0, 1, 0], [20, 3, 40], 4, 2, 128, seed=7, layers=3,
             layer=1)
    r.check(*r.call())
