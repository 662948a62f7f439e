"""A decoder layer with 8-bit integer products, from prefix to scores' input.

Builds a small store the way a deployment does offline (the selected states
of every document go through the layer's 8-bit key and value projections,
are normed and rotated, and enter the store), then runs the online tokens of
a batch of (query, document) pairs through the whole layer, once with bf16
products (``pipeline.LayerStep``) and once with 8-bit ones
(``pipeline.QuantLayerStep``), and prints both times and how far apart the
outputs are.  With --store fp4 the store holds the states in 4 bits, and the
keys are normed and rotated on their way into it.

    python3 -m paper_2609_03311_amd.quant_layer [--config qwen3_0p6b]
        [--pairs 800] [--tokens N] [--store bf16|fp4]

Weights and states are random (seeded); the shapes are the named workload's.
"""
from __future__ import annotations

import argparse

import numpy as np


def _time_ms(run, steps):
    import torch
    for _ in range(2):
        run()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(steps):
        run()
    end.record()
    torch.cuda.synchronize()
    return begin.elapsed_time(end) / steps


def main(argv=None):
    import torch

    import workloads
    from . import (DOPR_STORE_BF16, DOPR_STORE_FP4, dopr_check_status,
                   dopr_store_create, dopr_store_put)
    from .pipeline import LayerStep, QuantLayerStep, online_positions

    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", default="qwen3_0p6b",
                    choices=["tiny", "qwen3_0p6b", "qwen3_4b", "qwen3_8b"])
    ap.add_argument("--pairs", type=int, default=800)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--tokens", type=int, default=0,
                    help="online tokens of every pair (0: the workload's)")
    ap.add_argument("--store", default="bf16", choices=["bf16", "fp4"])
    args = ap.parse_args(argv)
    dev = "cuda"
    full = workloads.make(args.config)
    pairs = min(args.pairs, full.n_pairs)
    # the first pairs, over a store of just their documents
    docs, ids = np.unique(full.doc_ids[:pairs], return_inverse=True)
    seqlens = full.seqlens[:pairs]
    if args.tokens > 0:
        seqlens = np.full_like(seqlens, args.tokens)
    st = workloads.custom(full.doc_len[docs], ids.astype(np.int32), seqlens,
                          full.n_q_heads, full.n_kv_heads, name=args.config)
    hidden, inter = workloads.layer_dims(full)
    weights = workloads.layer_weights(st, hidden, inter, dev)
    prm = workloads.params(st, dev)
    x = workloads.hidden_states(st, hidden, dev)
    fp4 = args.store == "fp4"
    store = dopr_store_create(1, st.n_kv_heads, st.head_dim, st.doc_len,
                              device=dev, format=DOPR_STORE_FP4 if fp4
                              else DOPR_STORE_BF16)
    shape = dict(n_pairs=st.n_pairs, n_q_heads=st.n_q_heads,
                 total_tokens=st.n_tokens, max_tokens=int(st.seqlens.max()),
                 hidden=hidden, intermediate=inter, device=dev)
    quant = QuantLayerStep(store, weights, **shape)

    # offline: every document's selected states become stored keys and values
    cu = np.concatenate([[0], np.cumsum(st.doc_len, dtype=np.int64)])
    slots = int(cu[-1])
    gen = torch.Generator(device=dev).manual_seed(5)
    states = torch.randn((slots, hidden), generator=gen,
                         device=dev).to(torch.bfloat16)
    pos = torch.from_numpy((np.arange(slots) - np.repeat(cu[:-1], st.doc_len))
                           .astype(np.int32)).to(dev)
    ids = torch.arange(st.n_docs, dtype=torch.int32, device=dev)
    src_cu = torch.from_numpy(cu).to(dev)
    if fp4:
        quant.put_states(0, ids, src_cu, states, pos, prm["k_norm_w"])
    else:
        k, v = quant.prefix_states(states, pos, prm["k_norm_w"])
        dopr_store_put(store, 0, ids, src_cu, k, v)

    # online: the pairs' tokens through the layer
    doc_ids = torch.from_numpy(st.doc_ids).to(dev)
    cu_seqlens = torch.from_numpy(st.cu_seqlens).to(dev)
    positions = online_positions(st.doc_len, st.doc_ids, st.cu_seqlens, dev)
    norms = (prm["q_norm_w"], prm["k_norm_w"])
    bf16 = LayerStep(store, weights, **shape)
    t16 = _time_ms(lambda: bf16.run(0, doc_ids, cu_seqlens, x, *norms),
                   args.steps)
    t8 = _time_ms(lambda: quant.run(0, doc_ids, cu_seqlens, x, positions,
                                    *norms), args.steps)
    status = dopr_check_status(store)
    if status != 0:
        raise SystemExit(f"device status {status}")
    a, b = bf16.y.float(), quant.y.float()
    rel = ((a - b).pow(2).mean() / a.pow(2).mean()).sqrt().item()
    print(f"{args.config}: {st.n_pairs} pairs, {st.n_tokens} tokens, "
          f"{st.n_docs} documents, {slots} prefix slots")
    print(f"bf16 products {t16:.3f} ms, 8-bit products {t8:.3f} ms "
          f"({t16 / t8:.2f}x), relative RMS difference {rel:.4f}")
    return rel


if __name__ == "__main__":
    main()
