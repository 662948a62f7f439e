"""One decoder layer's online DoPR step on an HBM prefix store, and the
offline salience selection that decides what the store holds.

A thin convenience layer over the C ABI: it allocates device buffers with
torch and issues the library calls; all computation runs in the HIP kernels.
"""
from __future__ import annotations

import numpy as np

from . import (DOPR_STORE_BF16, dopr_decoder_layer,
               dopr_decoder_layer_workspace,
               dopr_norm_residual, dopr_prefix_attn, dopr_prefix_attn_score,
               dopr_prefix_attn_score_workspace, dopr_prefix_attn_workspace,
               dopr_quant_matmul, dopr_quant_matmul_workspace,
               dopr_quantize_rows, dopr_rotary, dopr_rotary_frequencies,
               dopr_salience, dopr_salience_workspace, dopr_score_logits,
               dopr_store_create, dopr_store_put, dopr_store_put_rotary)

HEAD_DIM = 128


def make_store(doc_len, n_kv_heads, k_src, v_src, *, n_layers=1, layer=0,
               device="cuda", stream=None, format=DOPR_STORE_BF16):
    """Create a store (of bf16 states, or DOPR_STORE_FP4) for `doc_len` and
    fill `layer` from canonical prefix states k_src/v_src [slots, Hkv, D]
    (bf16, device; D = 128 or 64) holding the resident documents' slots in
    ascending doc-id order."""
    import torch
    doc_len = np.ascontiguousarray(doc_len, np.int32)
    store = dopr_store_create(n_layers, n_kv_heads, int(k_src.shape[-1]),
                              doc_len, device=device, stream=stream,
                              format=format)
    res = np.nonzero(doc_len >= 0)[0].astype(np.int32)
    if res.size:
        cu = np.zeros(res.size + 1, np.int64)
        np.cumsum(doc_len[res], out=cu[1:])
        ids = torch.from_numpy(res).to(device)
        cu_t = torch.from_numpy(cu).to(device)
        dopr_store_put(store, layer, ids, cu_t, k_src, v_src, stream=stream)
    return store


class OnlineStep:
    """Reusable buffers for the per-batch step: prefix attention over the
    store, then the score head on each pair's score-token output row."""

    def __init__(self, store, *, n_pairs, n_q_heads, total_tokens,
                 max_tokens, kernel_variant=0, device="cuda", with_lse=False,
                 rows_per_item=0, queue_order=0):
        import torch
        self.store = store
        self.n_pairs = n_pairs
        self.n_q_heads = n_q_heads
        self.total_tokens = total_tokens
        self.max_tokens = max_tokens
        self.kernel_variant = kernel_variant
        self.rows_per_item = rows_per_item
        self.queue_order = queue_order
        nbytes = dopr_prefix_attn_workspace(
            store, n_pairs=n_pairs, n_q_heads=n_q_heads,
            max_tokens=max_tokens, total_tokens=total_tokens,
            kernel_variant=kernel_variant, rows_per_item=rows_per_item)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8,
                                     device=device)
        self.out = torch.empty((total_tokens, n_q_heads, store.head_dim),
                               dtype=torch.bfloat16, device=device)
        self.lse = (torch.empty((total_tokens, n_q_heads), dtype=torch.float32,
                                device=device) if with_lse else None)
        self.score = torch.empty(n_pairs, dtype=torch.float32, device=device)
        self.logits = torch.empty((n_pairs, 2), dtype=torch.float32,
                                  device=device)

    def attention(self, layer, doc_ids, cu_seqlens, q, k, v, q_norm_w,
                  k_norm_w, stream=None, **kw):
        dopr_prefix_attn(self.store, layer, doc_ids, cu_seqlens, q, k, v,
                         q_norm_w, k_norm_w, self.out, self.workspace,
                         max_tokens=self.max_tokens, lse=self.lse,
                         total_tokens=self.total_tokens,
                         kernel_variant=self.kernel_variant, stream=stream,
                         rows_per_item=self.rows_per_item,
                         **{"queue_order": self.queue_order, **kw})

    def score_head(self, cu_seqlens, norm_w, w_head, stream=None,
                   rms_eps=1e-6):
        width = self.n_q_heads * self.store.head_dim
        dopr_score_logits(self.out, norm_w, w_head, self.score, width=width,
                          h_row_stride=width, cu_seqlens=cu_seqlens,
                          logits=self.logits, rms_eps=rms_eps,
                          n_pairs=self.n_pairs, stream=stream)

    def run(self, layer, doc_ids, cu_seqlens, q, k, v, q_norm_w, k_norm_w,
            norm_w, w_head, stream=None):
        self.attention(layer, doc_ids, cu_seqlens, q, k, v, q_norm_w,
                       k_norm_w, stream=stream)
        self.score_head(cu_seqlens, norm_w, w_head, stream=stream)


class ScoreStep:
    """Reusable buffers for last-layer scoring: only each pair's score-token
    rows are attended, and the score head is fused into the attention
    epilogue.  `with_rows` keeps the rows (out [P, Hq, D], lse [P, Hq])."""

    def __init__(self, store, *, n_pairs, n_q_heads, total_tokens,
                 max_tokens, kernel_variant=0, device="cuda",
                 with_rows=True, queue_order=0):
        import torch
        self.store = store
        self.n_pairs = n_pairs
        self.n_q_heads = n_q_heads
        self.total_tokens = total_tokens
        self.max_tokens = max_tokens
        self.kernel_variant = kernel_variant
        self.queue_order = queue_order
        nbytes = dopr_prefix_attn_score_workspace(
            store, n_pairs=n_pairs, n_q_heads=n_q_heads,
            max_tokens=max_tokens, total_tokens=total_tokens,
            kernel_variant=kernel_variant)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8,
                                     device=device)
        self.out = (torch.empty((n_pairs, n_q_heads, store.head_dim),
                                dtype=torch.bfloat16, device=device)
                    if with_rows else None)
        self.lse = (torch.empty((n_pairs, n_q_heads), dtype=torch.float32,
                                device=device) if with_rows else None)
        self.score = torch.empty(n_pairs, dtype=torch.float32, device=device)
        self.logits = torch.empty((n_pairs, 2), dtype=torch.float32,
                                  device=device)

    def run(self, layer, doc_ids, cu_seqlens, q, k, v, q_norm_w, k_norm_w,
            norm_w, w_head, stream=None, **kw):
        dopr_prefix_attn_score(
            self.store, layer, doc_ids, cu_seqlens, q, k, v, q_norm_w,
            k_norm_w, self.out, self.workspace, norm_w, w_head, self.score,
            max_tokens=self.max_tokens, logits=self.logits, lse=self.lse,
            total_tokens=self.total_tokens,
            kernel_variant=self.kernel_variant, stream=stream,
            **{"queue_order": self.queue_order, **kw})


# names of the layer weights in the generator's dict -> the C struct fields
LAYER_KEYS = {"attn_norm": "attn_norm_w", "wq": "w_q", "wk": "w_k",
              "wv": "w_v", "wo": "w_o", "mlp_norm": "mlp_norm_w",
              "w_gate": "w_gate", "w_up": "w_up", "w_down": "w_down"}


class LayerStep:
    """Reusable buffers for one decoder layer over the online tokens:
    x [Ntok, W] in, y [Ntok, W] out, the layer's intermediates in one
    workspace."""

    def __init__(self, store, weights, *, n_pairs, n_q_heads, total_tokens,
                 max_tokens, hidden, intermediate, kernel_variant=0,
                 device="cuda", with_lse=False):
        import torch
        self.store = store
        self.weights = {LAYER_KEYS.get(k, k): v for k, v in weights.items()}
        self.n_q_heads = n_q_heads
        self.max_tokens = max_tokens
        self.hidden = hidden
        self.intermediate = intermediate
        self.kernel_variant = kernel_variant
        nbytes = dopr_decoder_layer_workspace(
            store, self.weights, n_pairs=n_pairs, n_q_heads=n_q_heads,
            max_tokens=max_tokens, total_tokens=total_tokens, hidden=hidden,
            intermediate=intermediate, kernel_variant=kernel_variant)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8,
                                     device=device)
        self.y = torch.empty((total_tokens, hidden), dtype=torch.bfloat16,
                             device=device)
        self.lse = (torch.empty((total_tokens, n_q_heads),
                                dtype=torch.float32, device=device)
                    if with_lse else None)

    def run(self, layer, doc_ids, cu_seqlens, x, q_norm_w, k_norm_w,
            stream=None, **kw):
        dopr_decoder_layer(self.store, layer, doc_ids, cu_seqlens, x, self.y,
                           self.weights, q_norm_w, k_norm_w, self.workspace,
                           n_q_heads=self.n_q_heads,
                           max_tokens=self.max_tokens, hidden=self.hidden,
                           intermediate=self.intermediate, lse=self.lse,
                           kernel_variant=self.kernel_variant, stream=stream,
                           **kw)


def online_positions(doc_len, doc_ids, cu_seqlens, device="cuda"):
    """Positions of a batch's online tokens, int32 [Ntok]: pair p's token j
    stands at L_d + j, behind its document's prefix."""
    import torch
    cu = np.asarray(cu_seqlens, np.int64)
    lens = np.diff(cu)
    ids = np.asarray(doc_ids, np.int64)
    doc_len = np.asarray(doc_len, np.int64)
    known = (ids >= 0) & (ids < doc_len.shape[0])
    first = np.where(known, np.maximum(doc_len[np.where(known, ids, 0)], 0), 0)
    pos = np.arange(int(cu[-1])) + np.repeat(first - cu[:-1], lens)
    return torch.from_numpy(pos.astype(np.int32)).to(device)


def quantize_weight(w):
    """A weight [out, in] in 8-bit integers with a scale per output channel:
    (int8 [out, in] on a row pitch of 16 bytes, fp32 [out])."""
    import torch
    out, width = w.shape
    pitch = -(-width // 16) * 16
    q = torch.empty((out, pitch), dtype=torch.int8, device=w.device)[:, :width]
    scale = torch.empty(out, dtype=torch.float32, device=w.device)
    dopr_quantize_rows(w, q, scale)
    return q, scale


class QuantLayerStep:
    """One decoder layer over the online tokens with 8-bit integer products:
    what LayerStep runs, with the projections' weights in 8 bits per output
    channel and their inputs in 8 bits per token, and with the layer's form
    open where families differ:

      rotary   dict(rotary_dim=, interleaved=, inv_freq=, attention_factor=),
               any of them: the rotation of q and k (default: rotate-half of
               the whole head at rope_theta, as LayerStep)
      weights  may hold post_attn_norm_w and post_mlp_norm_w [W] (a norm
               behind each block), attn_gate and mlp_gate [W] (a gain per
               channel on a block's output)
      residual_scale  on the residual stream at both joins

    x [Ntok, W] in, y [Ntok, W] out (bf16).  Weights are quantised once,
    here.  The MLP runs over `chunk` tokens at a time."""

    def __init__(self, store, weights, *, n_pairs, n_q_heads, total_tokens,
                 max_tokens, hidden, intermediate, rotary=None,
                 residual_scale=1.0, rope_theta=1e6, rms_eps=1e-6,
                 kernel_variant=0, chunk=32768, device="cuda"):
        import torch
        w = {LAYER_KEYS.get(k, k): v for k, v in weights.items()}
        d, hq, hk = store.head_dim, n_q_heads, store.n_kv_heads
        self.store = store
        self.n_q_heads, self.max_tokens = hq, max_tokens
        self.hidden, self.intermediate = hidden, intermediate
        self.residual_scale, self.rms_eps = residual_scale, rms_eps
        self.kernel_variant = kernel_variant
        self.norms = {k: w.get(k) for k in (
            "attn_norm_w", "mlp_norm_w", "post_attn_norm_w",
            "post_mlp_norm_w", "attn_gate", "mlp_gate")}
        # a plain second join rides in the down product
        self.plain_join = (w.get("post_mlp_norm_w") is None and
                           w.get("mlp_gate") is None and residual_scale == 1.0)
        self.w = {k: quantize_weight(w[k]) for k in ("w_q", "w_k", "w_v",
                                                     "w_o", "w_down")}
        self.w["w_gate_up"] = quantize_weight(
            torch.cat((w["w_gate"], w["w_up"])))
        r = dict(rotary or {})
        self.interleaved = bool(r.get("interleaved", False))
        self.attention_factor = float(r.get("attention_factor", 1.0))
        freq = r.get("inv_freq")
        if freq is None:
            freq, _ = dopr_rotary_frequencies(r.get("rotary_dim", d),
                                              rope_theta)
        self.inv_freq = freq.to(device)
        # the attention gets heads that are already normed and rotated
        self.no_rotation = torch.zeros(d // 2, dtype=torch.float32,
                                       device=device)
        n, c = total_tokens, min(total_tokens, chunk)
        self.chunk = max(c, 1)

        def bf16(*shape):
            return torch.empty(shape, dtype=torch.bfloat16, device=device)

        self.q, self.k = bf16(n, hq, d), bf16(n, hk, d)
        self.v, self.att = bf16(n, hk, d), bf16(n, hq, d)
        self.block, self.h, self.y = (bf16(n, hidden), bf16(n, hidden),
                                      bf16(n, hidden))
        self.gate_up = bf16(self.chunk, 2 * intermediate)
        self.x8 = self._int8(n, max(hidden, hq * d), device)
        self.a8 = self._int8(self.chunk, intermediate, device)
        self.x8_scale = torch.empty(n, dtype=torch.float32, device=device)
        self.a8_scale = torch.empty(self.chunk, dtype=torch.float32,
                                    device=device)
        last = n % self.chunk
        need = [dopr_quant_matmul_workspace(m, *self.w[k][0].shape)
                for k in self.w for m in {n, self.chunk, last}]
        self.product_ws = torch.empty(max(need + [256]), dtype=torch.uint8,
                                      device=device)
        nbytes = dopr_prefix_attn_workspace(
            store, n_pairs=n_pairs, n_q_heads=hq, max_tokens=max_tokens,
            total_tokens=n, kernel_variant=kernel_variant)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8,
                                     device=device)

    @staticmethod
    def _int8(rows, width, device):
        import torch
        return torch.empty((rows, -(-width // 16) * 16), dtype=torch.int8,
                           device=device)

    def _product(self, x8, scale, name, y, stream, **kw):
        w, w_scale = self.w[name]
        dopr_quant_matmul(x8, scale, w, w_scale, y, stream=stream,
                          workspace=self.product_ws, **kw)

    def _normed(self, x, gain, x8, scale, stream):
        """x8, scale = RMSNorm(x) * gain in 8 bits."""
        dopr_norm_residual(x, pre_norm_w=gain, q=x8, q_scale=scale,
                           rms_eps=self.rms_eps, stream=stream)

    def _prefix_products(self, x, stream):
        """The 8-bit key and value products of prefix inputs x."""
        import torch
        n, d, hk = x.shape[0], self.store.head_dim, self.store.n_kv_heads
        x8 = self._int8(n, self.hidden, x.device)[:, :self.hidden]
        scale = torch.empty(n, dtype=torch.float32, device=x.device)
        k, v = (torch.empty((n, hk, d), dtype=torch.bfloat16, device=x.device)
                for _ in range(2))
        need = dopr_quant_matmul_workspace(n, hk * d, self.hidden)
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
        self._normed(x, self.norms["attn_norm_w"], x8, scale, stream)
        for name, out in (("w_k", k), ("w_v", v)):
            w, w_scale = self.w[name]
            dopr_quant_matmul(x8, scale, w, w_scale, out.flatten(1),
                              workspace=ws, stream=stream)
        return k, v

    def prefix_states(self, x, positions, k_norm_w, stream=None):
        """Keys and values of this layer for prefix inputs x [slots, W] at
        `positions` (int32 [slots]): bf16 [slots, Hkv, D] each, the keys
        normed and rotated, as dopr_store_put takes them.  With a stream, they
        and the scratch in between are allocated on it."""
        import torch
        if stream is not None and stream != torch.cuda.current_stream():
            with torch.cuda.stream(stream):
                return self.prefix_states(x, positions, k_norm_w)
        k, v = self._prefix_products(x, stream)
        dopr_rotary(None, k, positions, self.inv_freq, None, k,
                    interleaved=self.interleaved,
                    attention_factor=self.attention_factor,
                    k_norm_w=k_norm_w, rms_eps=self.rms_eps, stream=stream)
        return k, v

    def put_states(self, layer, doc_ids, src_cu_slots, x, positions, k_norm_w,
                   stream=None):
        """The keys and values of prefix inputs x [slots, W] at `positions`
        into `layer` of the store, the keys normed and rotated on the way
        (dopr_store_put_rotary; doc_ids and src_cu_slots as there).  The
        scratch in between is allocated on `stream`."""
        import torch
        if stream is not None and stream != torch.cuda.current_stream():
            with torch.cuda.stream(stream):
                return self.put_states(layer, doc_ids, src_cu_slots, x,
                                       positions, k_norm_w)
        k, v = self._prefix_products(x, stream)
        dopr_store_put_rotary(self.store, layer, doc_ids, src_cu_slots, k, v,
                              self.inv_freq, positions=positions,
                              k_norm_w=k_norm_w, interleaved=self.interleaved,
                              attention_factor=self.attention_factor,
                              rms_eps=self.rms_eps, stream=stream)

    def run(self, layer, doc_ids, cu_seqlens, x, positions, q_norm_w=None,
            k_norm_w=None, stream=None, softmax_scale=None):
        n, W, I = x.shape[0], self.hidden, self.intermediate
        x8, scale = self.x8[:, :W], self.x8_scale
        self._normed(x, self.norms["attn_norm_w"], x8, scale, stream)
        for name, out in (("w_q", self.q), ("w_k", self.k), ("w_v", self.v)):
            self._product(x8, scale, name, out.flatten(1), stream)
        dopr_rotary(self.q, self.k, positions, self.inv_freq, self.q, self.k,
                    interleaved=self.interleaved,
                    attention_factor=self.attention_factor,
                    q_norm_w=q_norm_w, k_norm_w=k_norm_w,
                    rms_eps=self.rms_eps, stream=stream)
        dopr_prefix_attn(self.store, layer, doc_ids, cu_seqlens, self.q,
                         self.k, self.v, None, None, self.att, self.workspace,
                         max_tokens=self.max_tokens, total_tokens=n,
                         rms_eps=self.rms_eps, softmax_scale=softmax_scale,
                         kernel_variant=self.kernel_variant,
                         rope_inv_freq=self.no_rotation, stream=stream)
        att = self.att.flatten(1)
        a8 = self.x8[:, :att.shape[1]]
        dopr_quantize_rows(att, a8, scale, stream=stream)
        self._product(a8, scale, "w_o", self.block, stream)
        # the attention block joins the residual; the MLP's norm and 8 bits
        dopr_norm_residual(self.block, residual=x,
                           post_norm_w=self.norms["post_attn_norm_w"],
                           gate=self.norms["attn_gate"],
                           residual_scale=self.residual_scale,
                           pre_norm_w=self.norms["mlp_norm_w"], h=self.h,
                           q=x8, q_scale=scale, rms_eps=self.rms_eps,
                           stream=stream)
        for t0 in range(0, n, self.chunk):
            rows = slice(t0, min(t0 + self.chunk, n))
            m = rows.stop - t0
            gu = self.gate_up[:m]
            m8, m8_scale = self.a8[:m, :I], self.a8_scale[:m]
            self._product(x8[rows], scale[rows], "w_gate_up", gu, stream)
            dopr_quantize_rows(gu[:, :I], m8, m8_scale, up=gu[:, I:],
                               stream=stream)
            if self.plain_join:
                self._product(m8, m8_scale, "w_down", self.y[rows], stream,
                              residual=self.h[rows])
                continue
            self._product(m8, m8_scale, "w_down", self.block[rows], stream)
            dopr_norm_residual(self.block[rows], residual=self.h[rows],
                               post_norm_w=self.norms["post_mlp_norm_w"],
                               gate=self.norms["mlp_gate"],
                               residual_scale=self.residual_scale,
                               h=self.y[rows], rms_eps=self.rms_eps,
                               stream=stream)
        return self.y


class SalienceStep:
    """Reusable buffers for offline salience selection of a batch of
    documents: salience u of every token and the top-K_d positions of each
    document (K_d = n_d // ratio by default).  `with_attention` keeps the
    head-averaged attention of every document ([n_docs, M, M] fp32)."""

    def __init__(self, doc_lens, *, n_q_heads, n_kv_heads, top_p,
                 n_select=None, ratio=8, max_doclen=None, device="cuda",
                 with_attention=False):
        import torch
        lens = np.asarray(doc_lens, np.int64)
        self.n_docs = int(lens.shape[0])
        self.max_doclen = int(max_doclen or max(1, int(lens.max(initial=1))))
        self.top_p = top_p
        ks = (lens // ratio if n_select is None
              else np.asarray(n_select, np.int64))
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        cs = np.concatenate([[0], np.cumsum(ks)]).astype(np.int32)
        self.cu_host, self.cs_host = cu, cs
        self.cu = torch.from_numpy(cu).to(device)
        self.cs = torch.from_numpy(cs).to(device)
        ntok = int(cu[-1])
        self.u = torch.empty(ntok, dtype=torch.float32, device=device)
        self.selected = torch.empty(max(int(cs[-1]), 1), dtype=torch.int32,
                                    device=device)[:int(cs[-1])]
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        M = self.max_doclen
        self.attn_mean = (torch.empty((self.n_docs, M, M), dtype=torch.float32,
                                      device=device)
                          if with_attention else None)
        nbytes = dopr_salience_workspace(
            n_docs=self.n_docs, max_doclen=M, n_q_heads=n_q_heads,
            n_kv_heads=n_kv_heads, top_p=top_p, total_tokens=ntok,
            with_attention=with_attention)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8,
                                     device=device)

    def run(self, q, k, softmax_scale=HEAD_DIM ** -0.5, select=True,
            stream=None):
        dopr_salience(self.cu, q, k, self.u, max_doclen=self.max_doclen,
                      top_p=self.top_p, softmax_scale=softmax_scale,
                      cu_select=self.cs if select else None,
                      selected=self.selected if select else None,
                      attn_mean=self.attn_mean, status=self.status,
                      workspace=self.workspace, stream=stream)
