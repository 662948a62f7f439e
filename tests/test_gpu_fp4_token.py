"""Prefix attention of pairs of one token over a 4-bit store against the
definition in 64 bits.

What the kernel rounds: each softmax weight once to bf16 (2^-8 of itself, in
the weighted sum and in the normaliser alike) behind a logit whose query is
held in two bf16 parts (2^-16 of every product q_d k_d) and fp32 otherwise; the
own key's weight not at all; and the output once to bf16.  With A = sum of
weight * |value| and S = the largest sum of |q_d k_d| (natural-log units) of a
row, weights off by e = 2^-8 + 2^-14 S move the row by at most 2 e A, the
rounding by 2^-8 of the row, and the log-sum-exp by e."""
import numpy as np
import pytest
import torch

import fp4_refs

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _D():
    import paper_2609_03311_amd as D
    return D


class Tokens:
    def __init__(self, lens, docs, hq, hkv, d, *, norm=True, seed=0, scale=1.0,
                 gain=1.0, freq=True, layers=1, layer=0):
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
        self.q = randn(self.n, hq, d).to(torch.bfloat16)
        self.k = randn(self.n, hkv, d).to(torch.bfloat16)
        self.v = randn(self.n, hkv, d).to(torch.bfloat16)
        self.qw = self.kw = None
        if norm:
            self.qw, self.kw = ((gain * (1 + 0.1 * randn(d))).to(
                torch.bfloat16) for _ in range(2))
        self.freq = 1e6 ** (-torch.arange(0, d, 2).double() / d)
        self.given = self.freq.float().to(DEV) if freq else None
        if freq:
            self.freq = self.freq.float().double()
        self.cu = torch.arange(self.n + 1, dtype=torch.int32)

    def call(self, *, lse=True, variant=0, noalloc=False, cu=None, out=None,
             workspace=None, stream=None):
        D = _D()
        if out is None:
            out = torch.full((self.n, self.hq, self.d), 3.0,
                             dtype=torch.bfloat16, device=DEV)
        lse = torch.full((self.n, self.hq), 3.0, device=DEV) if lse else None
        on = [None if x is None else x.to(DEV) for x in
              (torch.tensor(self.docs, dtype=torch.int32),
               self.cu if cu is None else cu, self.q, self.k, self.v, self.qw,
               self.kw)]
        kw = dict(max_tokens=1, lse=lse, total_tokens=self.n,
                  rope_inv_freq=self.given, kernel_variant=variant,
                  stream=stream)
        if noalloc:
            D.dopr_prefix_attn_noalloc(self.store, self.layer, *on, out, **kw)
        else:
            if workspace is None:
                workspace = self.workspace(variant)
            D.dopr_prefix_attn(self.store, self.layer, *on, out, workspace,
                               **kw)
        return out, lse

    def workspace(self, variant=0):
        D = _D()
        need = D.dopr_prefix_attn_workspace(
            self.store, n_pairs=self.n, n_q_heads=self.hq, max_tokens=1,
            total_tokens=self.n, kernel_variant=variant)
        return torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)

    def check(self, out, lse, pairs=None):
        out, lse = out.cpu().double(), lse.cpu().double()
        scale = self.d ** -0.5
        for p in range(self.n) if pairs is None else pairs:
            doc = self.docs[p]
            if not 0 <= doc < len(self.lens) or self.lens[doc] < 0:
                assert (out[p] == 0).all()
                assert (lse[p] == -float("inf")).all()
                continue
            t = torch.tensor([float(self.lens[doc])]).double()

            def formed(x, w):
                x = x[p:p + 1].double()
                if w is not None:
                    x = x / torch.sqrt(x.square().mean(-1, keepdim=True)
                                       + 1e-6) * w.double()
                a, b = x[..., :self.d // 2], x[..., self.d // 2:]
                c, s = (t * self.freq).cos(), (t * self.freq).sin()
                return torch.cat((a * c - b * s, b * c + a * s), -1)[0]

            q, k = formed(self.q, self.qw), formed(self.k, self.kw)
            rep = self.hq // self.hkv
            r = self.rows[doc]
            keys = torch.cat((self.hk[r].double(), k[None]))   # [L+1, hkv, d]
            vals = torch.cat((self.hv[r].double(),
                              self.v[p:p + 1].double()))
            for g in range(self.hkv):
                qg = q[g * rep:(g + 1) * rep]
                x = qg @ keys[:, g].T * scale
                w = torch.softmax(x, -1)
                o, a = w @ vals[:, g], w @ vals[:, g].abs()
                size = (qg.abs() @ keys[:, g].abs().T * scale).amax(-1)
                e = (2.0 ** -8 + 2.0 ** -14 * size)[:, None]
                h = slice(g * rep, (g + 1) * rep)
                off = (out[p, h] - o).abs()
                assert (off <= 2.02 * e * a + 2.0 ** -8 * o.abs()
                        + 1e-30).all(), (p, g, off.max())
                want = torch.logsumexp(x, -1)
                assert ((lse[p, h] - want).abs() <= 1.01 * e[:, 0]
                        + 2.0 ** -20 * want.abs()).all(), (p, g)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (32, 8), (6, 2), (15, 3), (8, 1),
                                    (18, 2), (33, 1), (66, 2)])
@pytest.mark.parametrize("norm", [True, False])
def test_against_64_bits(d, hq, hkv, norm):
    lens = [0, 1, 31, 32, 33, 64, 100, 257, -1]
    docs = [0, 1, 2, 3, 4, 5, 6, 7, 8, 7, 3, 99, -1, 6]
    t = Tokens(lens, docs, hq, hkv, d, norm=norm, seed=hq + d, freq=norm)
    out, lse = t.call()
    t.check(out, lse)
    assert _D().dopr_check_status(t.store) == _D().DOPR_ERR_DOC_RANGE
    bare, none = t.call(lse=False)
    assert none is None and torch.equal(bare, out)
    other = t.call(noalloc=True)
    assert torch.equal(other[0], out) and torch.equal(other[1], lse)


@pytest.mark.parametrize("lens,docs,hq,hkv", [
    ([5000], [0], 8, 2), ([20001, 40], [0, 1, 0], 32, 8),
    ([513] * 7, list(range(7)), 3, 1), ([70001], [0], 40, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_long_prefixes_are_split(lens, docs, hq, hkv, d):
    t = Tokens(lens, docs, hq, hkv, d, seed=5)
    t.check(*t.call())


@pytest.mark.parametrize("scale,gain", [(40.0, 1.0), (1.0, 8.0),
                                        (2.0 ** -60, 1.0)])
@pytest.mark.parametrize("lens", [[40, 300, 0], [6000, 10, 3000]])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_of_any_size(scale, gain, lens, d):
    """Keys and gains over the reference-free range take the exact maximum."""
    t = Tokens(lens, [0, 1, 2, 0], 8, 2, d, seed=6, scale=scale, gain=gain)
    t.check(*t.call())


def test_layers_and_order_of_pairs():
    """The second of two layers, pairs in any order, all on one document."""
    t = Tokens([90], [0] * 40, 4, 2, 128, seed=7, layers=2, layer=1)
    t.check(*t.call())


def test_other_kernels_agree():
    """The planned kernels on the same call, to their roundings: one more of
    the query (2^-8 of every product), half a step of each output."""
    t = Tokens([300, 20], [0, 1, 1], 8, 2, 128, seed=8)
    out, lse = t.call()
    for variant in (8, 6, 4):
        o, l = t.call(variant=variant)
        assert (o.float() - out.float()).abs().max() < 0.05
        assert (l - lse).abs().max() < 0.05


def test_malformed_token_ranges():
    """Pairs of no token or of two are reported and left alone; the others
    run."""
    D = _D()
    t = Tokens([40, 33], [0, 1, 0, 1], 4, 2, 64, seed=9)
    want, _ = t.call()
    out = torch.full_like(want, 3.0)
    t.call(cu=torch.tensor([0, 1, 1, 3, 4], dtype=torch.int32), out=out)
    assert D.dopr_check_status(t.store) == D.DOPR_ERR_SEQLEN
    assert torch.equal(out[[0, 3]], want[[0, 3]])
    assert (out[[1, 2]] == 3.0).all()
    for bad in ([1, 2, 3, 4, 5], [0, 1, 2, 3, 5], [-1, 0, 1, 2, 3]):
        t.call(cu=torch.tensor(bad, dtype=torch.int32))
        assert D.dopr_check_status(t.store) == D.DOPR_ERR_SEQLEN


@pytest.mark.parametrize("lens", [[50, 300], [9000, 40]])
def test_graph_replays(lens):
    """A captured call, replayed with other inputs and eager work between."""
    t = Tokens(lens, [0, 1, 1, 0], 8, 2, 128, seed=10)
    D = _D()
    s = torch.cuda.Stream()
    bufs = [x.to(DEV) for x in (torch.tensor(t.docs, dtype=torch.int32),
                                t.cu, t.q, t.k, t.v, t.qw, t.kw)]
    out = torch.zeros((t.n, t.hq, t.d), dtype=torch.bfloat16, device=DEV)
    ws = t.workspace()

    def call():
        D.dopr_prefix_attn(t.store, 0, *bufs, out, ws, max_tokens=1,
                           total_tokens=t.n, rope_inv_freq=t.given,
                           stream=torch.cuda.current_stream())

    with torch.cuda.stream(s):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    for i in range(4):
        q = torch.randn(t.q.shape, generator=torch.Generator().manual_seed(i))
        t.q = q.to(torch.bfloat16)
        bufs[2].copy_(t.q)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want, _ = t.call()
        assert torch.equal(got, want), i


def test_grouping_takes_the_same_workspace():
    D = _D()
    t = Tokens([9, 4], [1, 0, 1], 2, 1, 128, seed=11)
    gd, gp, po = D.dopr_group_pairs(
        t.store, torch.tensor(t.docs, dtype=torch.int32, device=DEV),
        t.workspace())
    assert gd.tolist() == [0, 1] and gp.tolist() == [0, 1, 3]
    assert po.tolist() == [1, 0, 2]
