"""The operators of a 4-bit store as they are used together: states normed and
turned on their way in, attention of many tokens and of single ones over them,
the same states read back, copied and scored; and a layer that fills its store
so."""
import numpy as np
import pytest
import torch

import fp4_refs
import workloads
from test_gpu_fp4_rows import Rows, _same

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _D():
    import paper_2609_03311_amd as D
    return D


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


class Filled(Rows):
    """Rows over a store of two layers whose keys were normed and turned on
    the way in (held values from 64 bits)."""

    def __init__(self, lens, *args, layer=1, scale=1.0, seed=0, **kw):
        super().__init__(lens, *args, layers=2, layer=layer, seed=seed, **kw)
        D = _D()
        gen = torch.Generator().manual_seed(100 + seed)
        self.res = [i for i, n in enumerate(lens) if n >= 0]
        self.at = _cu([lens[i] for i in self.res])
        rows = int(self.at[-1])
        shape = (rows, self.hkv, self.d)
        self.raw = torch.randn(shape, generator=gen).to(torch.bfloat16)
        self.states = torch.randn(shape, generator=gen).to(torch.bfloat16)
        self.gain = (scale * (1 + 0.1 * torch.randn(
            self.d, generator=gen))).to(torch.bfloat16)
        self.given = self.freq.float().to(DEV)
        self.store = D.dopr_store_create(2, self.hkv, self.d,
                                         np.asarray(lens, np.int32),
                                         format=D.DOPR_STORE_FP4)
        self.put(self.gain)

    def put(self, gain, layer=None):
        D = _D()
        D.dopr_store_put_rotary(
            self.store, self.layer if layer is None else layer,
            torch.tensor(self.res, dtype=torch.int32, device=DEV),
            torch.from_numpy(self.at).to(DEV), self.raw.to(DEV),
            self.states.to(DEV), self.given, k_norm_w=gain.to(DEV))
        pos = torch.cat([torch.arange(b - a) for a, b in
                         zip(self.at[:-1], self.at[1:])])
        k = fp4_refs.turned_keys(self.raw, pos, self.given.cpu(), gain=gain)
        self.hk, self.hv = fp4_refs.held(k, self.states, self.at)

    def read(self):
        D = _D()
        k, v = (torch.full((int(self.at[-1]), self.hkv, self.d), 7.0,
                           dtype=torch.bfloat16, device=DEV)
                for _ in range(2))
        D.dopr_gather_prefix(
            self.store, self.layer,
            torch.tensor(self.res, dtype=torch.int32, device=DEV),
            torch.from_numpy(self.at).to(DEV), k, v)
        return k, v


@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 2), (64, 6, 2), (128, 3, 3)])
@pytest.mark.parametrize("tokens", ["many", "one"])
def test_fill_attend_read_copy(d, hq, hkv, tokens):
    D = _D()
    n = [1] * 9 if tokens == "one" else [5, 1, 40, 3, 2, 9, 33, 1, 70]
    r = Filled([70, 0, -1, 33, 2, 130], [0, 3, 5, 2, 1, 0, 4, 5, 3], n, hq,
               hkv, d, seed=len(n) + d)
    out, lse = r.call()
    r.check(out, lse)
    got = r.read()
    _same(got, (r.hk, r.hv))
    assert D.dopr_check_status(r.store) == D.DOPR_ERR_DOC_RANGE  # (doc 2)
    # a store without one of these documents, filled by a copy: the same bits
    lens = list(r.lens)
    lens[4] = -1
    fewer = D.dopr_store_create(2, hkv, d, np.asarray(lens, np.int32),
                                format=D.DOPR_STORE_FP4)
    D.dopr_store_copy_docs(fewer, r.store)
    mine, r.store = r.store, fewer
    less = r.call()
    r.store = mine
    a, b = int(r.cu[6]), int(r.cu[7])
    assert (less[0][a:b] == 0).all()
    for x, y in zip(less, (out, lse)):
        _same((x[:a], x[b:]), (y[:a], y[b:]))
    # a bf16 store of what was read: the block kernels give the same bits
    wide = D.dopr_store_create(2, hkv, d, np.asarray(r.lens, np.int32))
    D.dopr_store_put(wide, r.layer,
                     torch.tensor(r.res, dtype=torch.int32, device=DEV),
                     torch.from_numpy(r.at).to(DEV), *got)
    want = r.call(variant=8)
    r.store = wide
    _same(r.call(variant=8), want)


@pytest.mark.parametrize("tokens", [[1] * 5, [40, 3, 1, 17, 90]])
def test_smaller_keys_in_place_of_large_ones(tokens):
    """The logits' bound goes by the keys that are there now."""
    args = ([300, 20], [0, 1, 0, 1, 0], tokens, 8, 2, 128)
    fresh = Filled(*args, seed=3)
    want = fresh.call()
    again = Filled(*args, seed=3, scale=60.0)
    big, small = again.gain, fresh.gain
    assert big.abs().min() > 10 * small.abs().max()
    again.check(*again.call())
    again.put(small)
    again.call()
    _same(again.call(), want)
    again.check(*want)


@pytest.mark.parametrize("slots", [1024, 1025, 2047, 2100, 4200])
@pytest.mark.parametrize("tokens", [[1, 1, 1], [3, 1, 20]])
@pytest.mark.parametrize("d", [64, 128])
def test_joins_of_few_blocks(slots, tokens, d):
    r = Filled([slots, 40], [0, 1, 0], tokens, 6, 2, d, seed=slots)
    r.check(*r.call())


def test_two_streams_at_once():
    """Calls of two streams on one store, each with its own workspace, beside
    a put into the other layer."""
    r = Filled([90, 20, 400], [0, 1, 2, 0], [20, 3, 40, 1], 4, 2, 128, seed=8)
    one = Filled([90, 20, 400], [2, 1, 0, 2], [1] * 4, 4, 2, 128, seed=8)
    one.store = r.store
    want, single = r.call(), one.call()
    torch.cuda.synchronize()
    args = [(x, x.inputs(), x.workspace(), torch.cuda.Stream())
            for x in (r, one)]
    for _, _, _, s in args:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(5):
        got = []
        for x, inputs, ws, s in args:
            with torch.cuda.stream(s):
                got.append(x.call(inputs=inputs, workspace=ws, stream=s))
        r.put(r.gain, layer=0)
    torch.cuda.synchronize()
    _same(got[0], want)
    _same(got[1], single)


def test_graphs_that_share_a_workspace():
    """Two captured calls with one workspace, replayed by turns with eager
    work between."""
    D = _D()
    calls = [Filled([300, 20], [0, 1, 0], [40, 3, 90], 8, 2, 128, seed=4),
             Filled([300, 20], [1, 0], [1, 1], 8, 2, 128, seed=4),
             Filled([4000], [0], [2], 8, 2, 128, seed=5)]
    ws = max((x.workspace() for x in calls), key=lambda w: w.numel())
    s = torch.cuda.Stream()
    graphs, outs, want = [], [], []
    for x in calls:
        inputs = x.inputs()
        out = torch.zeros((x.total, x.hq, x.d), dtype=torch.bfloat16,
                          device=DEV)

        def call():
            D.dopr_prefix_attn(x.store, x.layer, *inputs, out, ws,
                               max_tokens=x.most, total_tokens=x.total,
                               rope_inv_freq=x.given,
                               stream=torch.cuda.current_stream())

        with torch.cuda.stream(s):
            call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        graphs.append((g, inputs))
        outs.append(out)
        want.append(x.call()[0])
    for _ in range(3):
        for (g, _), out, w in zip(graphs, outs, want):
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)
            calls[0].call(workspace=ws)


@pytest.mark.parametrize("tokens", [[1] * 4, [5, 40, 3, 17], [90] * 4])
@pytest.mark.parametrize("pairs", [1, 70])
def test_values_that_are_not_finite(tokens, pairs):
    """A pair's own keys and values leave other pairs' rows alone, and a
    document's the rows over other documents; keys that a mask hides change
    nothing before them."""
    lens, docs = [40, 70, 33], [0, 1, 0, 2] * pairs
    args = (lens, docs, tokens * pairs, 4, 2, 128)
    r = Filled(*args, seed=6)
    out, lse = r.call()
    rows = [(int(a), int(b)) for a, b in zip(r.cu[:-1], r.cu[1:])]
    a, b = rows[1]
    r.v[b - 1, 0, 5] = float("inf")
    r.k[b - 1, 1, 7] = float("nan")
    got, got_lse = r.call()
    keep = torch.ones(r.total, dtype=torch.bool)
    keep[a:b] = False
    _same((got[keep], got_lse[keep]), (out[keep], lse[keep]))
    # the first kv head's rows: one dim that is not finite, the rest as before
    mine, dims = got[a:b, :2].float(), torch.arange(128) != 5
    assert not torch.isfinite(mine[-1, :, 5]).any()
    _same((got[a:b, :2][..., dims],), (out[a:b, :2][..., dims],))
    # the second's: the token with the key, and none before
    assert torch.isnan(got[b - 1, 2:].float()).all()
    _same((got[a:b - 1, 2:],), (out[a:b - 1, 2:],))
    # a stored value: its dim, over its document
    r = Filled(*args, seed=6)
    r.states[41, 1, 9] = float("nan")  # (the second document's second slot)
    r.put(r.gain)
    got, _ = r.call()
    of = torch.zeros(r.total, dtype=torch.bool)
    for p, (a, b) in enumerate(rows):
        of[a:b] = docs[p] == 1
    hit = torch.zeros((r.total, 4, 128), dtype=torch.bool)
    hit[of, 2:, 9] = True
    assert torch.equal(torch.isnan(got.cpu().float()), hit)
    _same((got.cpu()[~hit],), (out.cpu()[~hit],))


def _step(fmt, **rotary):
    from paper_2609_03311_amd import dopr_store_create, pipeline
    st = workloads.custom(np.array([70, 5, 33], np.int32),
                          np.array([0, 2, 1], np.int32),
                          np.array([4, 1, 9], np.int32), 4, 2, name="small")
    w = workloads.layer_weights(st, 256, 512, DEV)
    store = dopr_store_create(1, st.n_kv_heads, st.head_dim, st.doc_len,
                              format=fmt)
    return st, store, pipeline.QuantLayerStep(
        store, w, n_pairs=st.n_pairs, n_q_heads=st.n_q_heads,
        total_tokens=st.n_tokens, max_tokens=int(st.seqlens.max()),
        hidden=256, intermediate=512, rotary=rotary or None)


@pytest.mark.parametrize("interleaved,r", [(False, 128), (True, 64)])
@pytest.mark.parametrize("other_stream", [False, True])
def test_a_layer_fills_its_store(interleaved, r, other_stream):
    """QuantLayerStep.put_states: a bf16 store holds what prefix_states gives,
    keys by one rounding less (two roundings of 2^-8 and fp32's against one);
    a 4-bit store the held values of its own products' keys."""
    D = _D()
    held = {}
    for fmt in (D.DOPR_STORE_BF16, D.DOPR_STORE_FP4):
        st, store, step = _step(fmt, rotary_dim=r, interleaved=interleaved)
        prm = workloads.params(st, DEV)
        cu = _cu(st.doc_len)
        x = torch.randn((int(cu[-1]), 256), generator=torch.Generator()
                        .manual_seed(2)).to(DEV, torch.bfloat16)
        pos = torch.cat([torch.arange(n) for n in st.doc_len]).to(
            DEV, torch.int32)
        ids = torch.arange(st.n_docs, dtype=torch.int32, device=DEV)
        at = torch.from_numpy(cu).to(DEV)
        s = torch.cuda.Stream() if other_stream else None
        if s is not None:
            s.wait_stream(torch.cuda.current_stream())
        step.put_states(0, ids, at, x, pos, prm["k_norm_w"], stream=s)
        torch.cuda.synchronize()
        k, v = (torch.empty((int(cu[-1]), st.n_kv_heads, 128),
                            dtype=torch.bfloat16, device=DEV)
                for _ in range(2))
        D.dopr_gather_prefix(store, 0, ids, at, k, v)
        held[fmt] = (k, v)
        pk, pv = step.prefix_states(x, pos, prm["k_norm_w"])
        if fmt == D.DOPR_STORE_BF16:
            _same((v,), (pv,))
            # (a rotation's two products, each of a factor off by 2^-24 three
            # times at most, next to a rounding of the sum on either side)
            part = pk.float().norm(dim=-1, keepdim=True)
            off = (k.float() - pk.float()).abs()
            assert (off <= 2.0 ** -7 * pk.float().abs()
                    + 2.0 ** -21 * part).all()
    wk, wv = fp4_refs.held(*(t.cpu() for t in held[D.DOPR_STORE_BF16]), cu)
    _same(held[D.DOPR_STORE_FP4], (wk, wv))


def test_a_layer_over_its_store():
    """Both layer steps over a 4-bit store that the layer filled."""
    from paper_2609_03311_amd import quant_layer
    assert quant_layer.main(["--config", "tiny", "--pairs", "20", "--steps",
                             "2", "--store", "fp4"]) <= 5e-2
