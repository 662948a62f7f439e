"""A prefix store held in 4 bits, as measurable cases.

Three operators: prefix states on their way into a store, their keys normed
and given their rotary positions (``dopr_store_put_rotary``, into a store of
``DOPR_STORE_FP4`` or bf16 states), the prefix attention over a 4-bit store
(``dopr_prefix_attn``), and the same attention for pairs of a single token.
The shapes are those of the repository's own workloads (32 q / 8 kv heads of
128, 129 online tokens, documents of 32 to 2048 slots, ragged batches, head
size 64 without QK-norm) and odd ones.

A 4-bit store holds blocks of 32 values: a 4-bit float (0, 0.5, 1, 1.5, 2, 3,
4, 6 and their negatives) times the block's power of two, the smallest 2^e
with 7 * 2^e at least the block's largest magnitude (e in -125 .. 125); a
value goes to the nearest, ties to the even code.  A key's block is the 32
dims 64 j + 16 i + 8 h + e of one (j, h), i < 4, e < 8, of one slot; a
value's block is one dim of 32 consecutive slots, from the document's first
(fewer at its end).

``run`` computes a case with elementary torch operations, or, with ``own``
set, through the library's entry points.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
THETA = 1e6


def _put(name, docs, slots, heads, head_dim, rotated, dtype="bf16", least=0,
         norm=False, interleaved=False, fused=0, fmt="fp4", first=0):
    """`docs` documents of `least` (0: all the same) to `slots` slots; fused:
    q heads beside k and v in one buffer's rows (0: k and v apart)."""
    return {"name": name, "kind": "put", "docs": docs, "slots": slots,
            "least": least, "kv_heads": heads, "head_dim": head_dim,
            "rotated": rotated, "dtype": dtype, "norm": norm,
            "interleaved": interleaved, "fused": fused, "format": fmt,
            "first": first}


def _attn(name, pairs, docs, tokens, slots, heads, head_dim, norm,
          least_tokens=0, least_slots=0, absent=0):
    """`pairs` pairs of `least_tokens` to `tokens` tokens over `docs`
    documents of `least_slots` to `slots` slots (0: all the same); `absent`
    of the pairs name a document that is not resident."""
    return {"name": name, "kind": "attn", "pairs": pairs, "docs": docs,
            "tokens": tokens, "least_tokens": least_tokens, "slots": slots,
            "least_slots": least_slots, "q_heads": heads[0],
            "kv_heads": heads[1], "head_dim": head_dim, "norm": norm,
            "absent": absent}


def listed():
    return [
        # one short document: the latency of putting states into a store
        _put("put_one_document", 1, 32, 8, 128, 128, norm=True),
        # fp16, three kv heads of 64, half of each rotated in the
        # interleaved layout, documents of any length from 1 slot on
        _put("put_odd", 301, 255, 3, 64, 32, "f16", least=1,
             interleaved=True, first=7),
        # a collection's documents out of one q, k, v buffer, normed: the
        # offline pass that fills a layer of the store
        _put("put_collection", 1024, 256, 8, 128, 128, norm=True, fused=32),
        # one pair's 129 online tokens on 256 prefix slots: latency
        _attn("attn_one_pair", 1, 1, 129, 256, (32, 8), 128, True),
        # one query's 100 candidates
        _attn("attn_one_query", 100, 100, 129, 256, (32, 8), 128, True),
        # ragged pairs that share documents, one document missing
        _attn("attn_ragged", 512, 300, 129, 255, (32, 8), 128, True, 17, 8,
              absent=1),
        # few tokens on long prefixes, head size 64, no QK-norm
        _attn("attn_long", 64, 16, 33, 4096, (32, 8), 64, False),
        # sixteen queries' candidates: the largest
        _attn("attn_many", 1600, 1000, 129, 256, (32, 8), 128, True),
        # one token of one pair: latency
        _attn("token_one", 1, 1, 1, 256, (32, 8), 128, True),
        # one token of one query's candidates on 1024 slots
        _attn("token_one_query", 100, 100, 1, 1024, (32, 8), 128, True),
        # one token on two very long prefixes: the slots have to be split
        _attn("token_long", 2, 2, 1, 50001, (32, 8), 128, True),
        # single tokens of thousands of pairs, ragged, some documents shared
        _attn("token_many", 4096, 3000, 1, 512, (32, 8), 128, True, 0, 64),
    ]


MOST_LOGITS = 1600 * 32 * 129 * 385    # pairs x heads x tokens x keys
MOST_STATES = 4096 * 512 * 8 * 128     # pairs x slots x heads x dims
MOST_PUT = 1024 * 256 * 8 * 128


def _log_int(rng, lo, hi):
    if hi <= lo:
        return lo
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["put", "attn", "token"], [30, 40, 30])[0]
    head_dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 8, 8, 8])
    if kind == "put":
        slots = _log_int(rng, 1, 2048)
        docs = _log_int(rng, 1, max(1, MOST_PUT // (slots * kv * head_dim)))
        docs = min(docs, 20000)
        rotated = rng.choice([head_dim, head_dim, head_dim // 2,
                              2 * rng.randint(1, head_dim // 2)])
        case = _put("", docs, slots, kv, head_dim, rotated,
                    rng.choice(["bf16", "bf16", "f16", "f32"]),
                    rng.choice([0, rng.randint(1, slots)]),
                    rng.random() < 0.5, rng.random() < 0.4,
                    rng.choice([0, kv, 4 * kv]),
                    rng.choice(["fp4", "fp4", "fp4", "bf16"]),
                    rng.choice([0, rng.randint(0, 4096)]))
    else:
        rep = rng.choice([1, 2, 3, 4, 4, 5, 8])
        slots = _log_int(rng, 1, 4096 if kind == "attn" else 50001)
        tokens = 1 if kind == "token" else _log_int(rng, 2, 257)
        most = min(MOST_LOGITS // (kv * rep * tokens * (slots + tokens)),
                   MOST_STATES // (slots * kv * head_dim))
        pairs = _log_int(rng, 1, max(1, min(most, 4096)))
        docs = rng.choice([pairs, max(1, pairs * 2 // 3),
                           max(1, pairs // 8)])
        case = _attn("", pairs, docs, tokens, slots, (kv * rep, kv),
                     head_dim, rng.random() < 0.6,
                     rng.choice([0, rng.randint(1, tokens)]),
                     rng.choice([0, rng.randint(0, slots)]),
                     0 if pairs < 8 else rng.choice([0, 0, 1]))
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# Inputs

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def _lengths(rng, n, least, most):
    """n lengths spread evenly over least .. most, in any order."""
    if not least:
        return np.full(n, most, np.int64)
    if n == 1:
        return np.array([most], np.int64)
    v = np.rint(np.linspace(least, most, n)).astype(np.int64)
    return rng.permutation(v)


def _offsets(lengths):
    out = np.zeros(lengths.size + 1, np.int64)
    np.cumsum(lengths, out=out[1:])
    return out


def _on(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def _frequencies(rotated):
    i = torch.arange(0, rotated, 2, dtype=torch.float64)
    return (THETA ** (-i / rotated)).float().to(DEV)


def _channels(gen, heads, head_dim):
    """Scales of a head's channels: a few run larger than the others, as in
    keys of trained models."""
    big = torch.rand((heads, head_dim), generator=gen, device=DEV) < 0.02
    return torch.where(big, 3.0, 1.0)


def _sources(case, seed):
    """Everything the two ways and the definition share: the documents'
    states before they are stored, and the batch."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    h, d = case["kv_heads"], case["head_dim"]
    s = dict(case)
    if case["kind"] == "put":
        dt = TYPES[case["dtype"]]
        lens = _lengths(rng, case["docs"], case["least"], case["slots"])
        cu = _offsets(lens)
        rows, hq = int(cu[-1]), case["fused"]
        if hq:
            buf = _randn(gen, rows, (hq + 2 * h) * d).to(dt)
            s["k"] = buf[:, hq * d:(hq + h) * d].view(rows, h, d)
            s["v"] = buf[:, (hq + h) * d:].view(rows, h, d)
        else:
            s["k"] = (_randn(gen, rows, h, d) * _channels(gen, h, d)).to(dt)
            s["v"] = _randn(gen, rows, h, d).to(dt)
        s["k_w"] = ((1.0 + 0.1 * _randn(gen, d)).to(dt) if case["norm"]
                    else None)
        s["inv_freq"] = _frequencies(case["rotated"])
        within = np.arange(rows) - np.repeat(cu[:-1], lens)
        s["positions"] = _on(within + case["first"], torch.int32)
        s["doc_len"], s["cu_host"] = lens.astype(np.int32), cu
        s["ids"] = torch.arange(case["docs"], dtype=torch.int32, device=DEV)
        s["cu"] = _on(cu, torch.int64)
        return s
    p, n = case["pairs"], case["docs"]
    lens = _lengths(rng, n, case["least_slots"], case["slots"])
    cu = _offsets(lens)
    rows = int(cu[-1])
    s["k_src"] = (_randn(gen, rows, h, d)
                  * _channels(gen, h, d)).to(torch.bfloat16)
    s["v_src"] = _randn(gen, rows, h, d).to(torch.bfloat16)
    # (an absent document is the last id; every other one is named)
    ids = np.concatenate([np.arange(n), rng.integers(0, n, p - n)])
    ids = rng.permutation(ids)
    if case["absent"]:
        at = rng.choice(p, case["absent"], replace=False)
        ids[at] = n
    toks = _lengths(rng, p, case["least_tokens"], case["tokens"])
    s["doc_len"] = np.append(lens, -1).astype(np.int32)
    s["cu_host"] = cu
    s["doc_ids"] = _on(ids, torch.int32)
    tcu = _offsets(toks)
    s["cu_seqlens"] = _on(tcu, torch.int32)
    total, hq = int(tcu[-1]), case["q_heads"]
    s["q"] = _randn(gen, total, hq, d).to(torch.bfloat16)
    s["k"] = _randn(gen, total, h, d).to(torch.bfloat16)
    s["v"] = _randn(gen, total, h, d).to(torch.bfloat16)
    s["q_w"] = s["k_w"] = None
    if case["norm"]:
        s["q_w"], s["k_w"] = ((1.0 + 0.1 * _randn(gen, d)).to(torch.bfloat16)
                              for _ in range(2))
    s["inv_freq"] = _frequencies(d)
    return s


def prepare(case, seed):
    s = _sources(case, seed)
    h, d = case["kv_heads"], case["head_dim"]
    if case["kind"] == "put":
        s["k_out"] = torch.empty((s["k"].shape[0], h, d),
                                 dtype=torch.bfloat16, device=DEV)
        s["v_out"] = torch.empty_like(s["k_out"])
        if own:
            import paper_2609_03311_amd as D
            s["store"] = D.dopr_store_create(
                1, h, d, s["doc_len"],
                format=(D.DOPR_STORE_FP4 if case["format"] == "fp4"
                        else D.DOPR_STORE_BF16))
        return s
    k, v = s.pop("k_src"), s.pop("v_src")
    n = case["docs"]
    cu = _on(s["cu_host"], torch.int64)
    s["out"] = torch.empty_like(s["q"])
    if own:
        import paper_2609_03311_amd as D
        s["store"] = D.dopr_store_create(1, h, d, s["doc_len"],
                                         format=D.DOPR_STORE_FP4)
        ids = torch.arange(n, dtype=torch.int32, device=DEV)
        D.dopr_store_put(s["store"], 0, ids, cu, k, v)
        need = D.dopr_prefix_attn_workspace(
            s["store"], n_pairs=case["pairs"], n_q_heads=case["q_heads"],
            max_tokens=case["tokens"], total_tokens=s["q"].shape[0])
        s["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8,
                                     device=DEV)
        torch.cuda.synchronize()
    else:
        # the plain form's cache: documents on one stride, two codes a byte,
        # exponents beside them
        at, there = _padded(cu, -(-case["slots"] // 32) * 32)
        k, e = _encode_keys(_spread(k, at, there).float())
        s["k_codes"], s["k_exp"] = _pack(k), e
        v, e = _encode_values(_spread(v, at, there).float())
        s["v_codes"], s["v_exp"] = _pack(v), e
        s["lens"] = _on(s["doc_len"], torch.int64)
    return s


# ---------------------------------------------------------------------------
# The 4-bit form in elementary operations

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _padded(cu, width):
    """Row of each (document, slot) of `width` slots, and which there are."""
    lens = cu[1:] - cu[:-1]
    j = torch.arange(width, device=DEV)
    there = j[None, :] < lens[:, None]
    return torch.where(there, cu[:-1, None] + j[None, :], 0), there


def _spread(x, at, there):
    return x[at] * there[..., None, None].to(x.dtype)


def _power(e):
    """2^e in 32 bits, exactly, for e in -126 .. 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(b):
    """Blocks b [..., 32] -> codes 0 .. 15 and exponents [...]."""
    a = b.abs().amax(-1)
    m, e = torch.frexp(a)
    e = torch.where(m > 0.875, e - 2, e - 3)
    e = torch.where(a > 0, e, -125).clamp(-125, 125)
    t = b.abs() * _power(-e[..., None])
    c = ((t > 0.25).byte() + (t >= 0.75).byte() + (t > 1.25).byte()
         + (t >= 1.75).byte() + (t > 2.5).byte() + (t >= 3.5).byte()
         + (t > 5.0).byte())
    return c + 8 * torch.signbit(b).byte(), e.to(torch.int8)


def _decode(codes, e):
    table = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=DEV)
    return table[codes.int()] * _power(e[..., None])


def _key_blocks(x):
    """[..., D] -> [..., D / 32, 32] by the blocks of a key."""
    *lead, d = x.shape
    x = x.reshape(*lead, d // 64, 4, 2, 8).transpose(-3, -2)
    return x.reshape(*lead, d // 32, 32)


def _keys_of(b):
    *lead, n, _ = b.shape
    b = b.reshape(*lead, n // 2, 2, 4, 8).transpose(-3, -2)
    return b.reshape(*lead, 32 * n)


def _value_blocks(x):
    """[n, L, H, D] -> [n, L / 32, H, D, 32]"""
    n, width, h, d = x.shape
    return x.reshape(n, width // 32, 32, h, d).permute(0, 1, 3, 4, 2)


def _values_of(b):
    n, m, h, d, _ = b.shape
    return b.permute(0, 1, 4, 2, 3).reshape(n, 32 * m, h, d)


def _encode_keys(x):
    return _encode(_key_blocks(x))


def _encode_values(x):
    return _encode(_value_blocks(x))


def _pack(codes):
    return codes[..., 0::2] + 16 * codes[..., 1::2]


def _unpack(packed):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2)


# ---------------------------------------------------------------------------
# One pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2609_03311_amd as D
    if s["kind"] == "put":
        D.dopr_store_put_rotary(s["store"], 0, s["ids"], s["cu"], s["k"],
                                s["v"], s["inv_freq"],
                                positions=s["positions"], k_norm_w=s["k_w"],
                                interleaved=s["interleaved"], rms_eps=EPS)
        D.dopr_gather_prefix(s["store"], 0, s["ids"], s["cu"], s["k_out"],
                             s["v_out"])
        return s["k_out"], s["v_out"]
    D.dopr_prefix_attn(s["store"], 0, s["doc_ids"], s["cu_seqlens"], s["q"],
                       s["k"], s["v"], s["q_w"], s["k_w"], s["out"],
                       s["workspace"], max_tokens=s["tokens"], rms_eps=EPS,
                       rope_inv_freq=s["inv_freq"])
    return s["out"]


def _rms_norm(v, gain):
    inv = 1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * inv * gain.to(v.dtype)


def _rotate(x, angle, rotated, interleaved):
    """x [rows, heads, D] turned by angle [rows, rotated / 2]."""
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    if interleaved:
        a, b = x[..., 0:rotated:2], x[..., 1:rotated:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1)
        turned = turned.flatten(-2)
    else:
        a, b = x[..., :rotated // 2], x[..., rotated // 2:rotated]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., rotated:]), -1)


def _run_plain(s):
    return _put_plain(s) if s["kind"] == "put" else _attn_plain(s)


def _put_plain(s):
    # in 64 bits: a key next to the border of two codes goes to the right one
    k = s["k"].double()
    if s["k_w"] is not None:
        k = _rms_norm(k, s["k_w"])
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()[None]
    k = _rotate(k, angle, s["rotated"], s["interleaved"]).to(torch.bfloat16)
    v = s["v"].to(torch.bfloat16)
    if s["format"] == "bf16":
        return k, v
    k = _keys_of(_decode(*_encode_keys(k.float())))
    at, there = _padded(s["cu"], -(-s["slots"] // 32) * 32)
    v = _values_of(_decode(*_encode_values(_spread(v, at, there).float())))
    return k.to(torch.bfloat16), v[there].to(torch.bfloat16)


def _attn_plain(s):
    kc = _keys_of(_decode(_unpack(s["k_codes"]), s["k_exp"]))
    vc = _values_of(_decode(_unpack(s["v_codes"]), s["v_exp"]))
    n, width, h, d = kc.shape
    p, hq = s["pairs"], s["q_heads"]
    rep, t = hq // h, s["tokens"]
    doc, cu = s["doc_ids"].long(), s["cu_seqlens"].long()
    slots = s["lens"][doc]                              # -1: not resident
    doc = doc.clamp(max=n - 1)
    # q and k of every token, normed and turned behind its prefix
    total = s["q"].shape[0]
    pair = torch.repeat_interleave(torch.arange(p, device=DEV),
                                   cu[1:] - cu[:-1], output_size=total)
    pos = slots[pair] + torch.arange(total, device=DEV) - cu[pair]
    angle = pos.double()[:, None] * s["inv_freq"].double()[None]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if s["q_w"] is not None:
        q, k = _rms_norm(q, s["q_w"]), _rms_norm(k, s["k_w"])
    turn = torch.polar(torch.ones_like(angle), angle)
    cos, sin = turn.real.float()[:, None], turn.imag.float()[:, None]

    def turned(x):
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)

    q, k = turned(q), turned(k)
    # pairs on one stride: [pair, kv head, tokens x q heads, D]
    at, there = _padded(cu, t)
    q = q[at].reshape(p, t, h, rep, d).permute(0, 2, 1, 3, 4)
    q = q.reshape(p * h, t * rep, d) * d ** -0.5
    keys = torch.cat((kc[doc], k[at]), 1)               # [p, width + t, h, d]
    keys = keys.permute(0, 2, 3, 1).reshape(p * h, d, width + t).contiguous()
    logits = torch.bmm(q, keys).view(p, h, t, rep, width + t)
    del keys
    j = torch.arange(width, device=DEV)
    step = torch.arange(t, device=DEV)
    seen = torch.cat((
        (j[None, None, :] < slots[:, None, None]).expand(p, t, width),
        (step[None, None, :] <= step[None, :, None])
        & there[:, None, :]), -1)
    logits.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    logits -= logits.amax(-1, keepdim=True)
    w = logits.exp_()
    w /= w.sum(-1, keepdim=True)
    values = torch.cat((vc[doc], v[at]), 1).permute(0, 2, 1, 3)
    values = values.reshape(p * h, width + t, d).contiguous()
    o = torch.bmm(w.view(p * h, t * rep, width + t), values)
    o = o.view(p, h, t, rep, d).permute(0, 2, 1, 3, 4).reshape(p, t, hq, d)
    o = torch.where((slots >= 0)[:, None, None, None], o, 0.0)
    return o[there].to(torch.bfloat16)


# ---------------------------------------------------------------------------
# The definition in 64 bits, written apart from the plain form

def _power64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _held(blocks):
    """What the blocks [n, 32] (bf16 values) stand for once held in 4 bits."""
    b = blocks.double()
    a = b.abs().max(1, keepdim=True).values
    unit = _power64(torch.ceil(torch.log2(a / 7.0)).clamp(-126, 126))
    # (the logarithm may be off next to a power of two)
    unit = torch.where(a <= 3.5 * unit, unit / 2, unit)
    unit = torch.where(a > 7.0 * unit, unit * 2, unit)
    unit = unit.clamp(2.0 ** -125, 2.0 ** 125)
    t = b.abs() / unit
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0],
                        dtype=torch.float64, device=b.device)
    low = torch.bucketize(t, mids, out_int32=True)
    high = torch.bucketize(t, mids, out_int32=True, right=True)
    code = torch.where(low % 2 == 0, low, high)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=b.device)
    return torch.copysign(level[code.long()] * unit, b)


def _held_keys(k):
    rows, h, d = k.shape
    dim = torch.arange(d, device=k.device)
    # dims by block: (dim / 64, (dim / 8) % 2), then by place in it
    order = torch.argsort((dim // 64) * 2 + (dim // 8) % 2, stable=True)
    out = torch.empty(k.shape, dtype=torch.float64, device=k.device)
    out[..., order] = _held(k[..., order].reshape(-1, 32)).view(rows, h, d)
    return out


def _held_values(v, cu):
    """v [slots, H, D] of documents at cu (host), in one go: every document
    filled up to whole blocks with zeros."""
    rows, h, d = v.shape
    lens = np.diff(cu)
    whole = -(-lens // 32) * 32
    to = np.repeat(_offsets(whole)[:-1], lens)
    to = _on(to + np.arange(rows) - np.repeat(cu[:-1], lens), torch.int64)
    wide = torch.zeros((int(whole.sum()), h, d), dtype=v.dtype,
                       device=v.device)
    wide[to] = v
    b = wide.view(-1, 32, h * d).transpose(1, 2)
    held = _held(b.reshape(-1, 32)).view(-1, h * d, 32).transpose(1, 2)
    return held.reshape(-1, h, d)[to]


def _turn64(x, gain, angle, rotated, interleaved):
    x = x.double()
    if gain is not None:
        power = x.square().sum(-1, keepdim=True) / x.shape[-1]
        x = x * torch.rsqrt(power + EPS) * gain.double()
    i = torch.arange(rotated // 2, device=x.device)
    one = 2 * i if interleaved else i
    two = one + 1 if interleaved else i + rotated // 2
    z = torch.complex(x[..., one], x[..., two])
    z = z * torch.polar(torch.ones_like(angle), angle).unsqueeze(1)
    out = x.clone()
    out[..., one], out[..., two] = z.real, z.imag
    return out


def exact(case, seed):
    s = _sources(case, seed)
    freq = s["inv_freq"].double()
    if case["kind"] == "put":
        angle = s["positions"].double().unsqueeze(1) * freq
        k = _turn64(s["k"], s["k_w"], angle, case["rotated"],
                    case["interleaved"])
        k, v = k.to(torch.bfloat16), s["v"].to(torch.bfloat16)
        if case["format"] == "bf16":
            return k.double(), v.double()
        return _held_keys(k), _held_values(v, s["cu_host"])
    kc = _held_keys(s["k_src"])
    vc = _held_values(s["v_src"], s["cu_host"])
    d, hk, hq = case["head_dim"], case["kv_heads"], case["q_heads"]
    cu = s["cu_seqlens"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for i, doc in enumerate(s["doc_ids"].tolist()):
        length = int(s["doc_len"][doc])
        if length < 0:
            continue
        a, t = cu[i], cu[i + 1] - cu[i]
        angle = (length + torch.arange(t, device=DEV)).double()
        angle = angle.unsqueeze(1) * freq
        q = _turn64(s["q"][a:a + t], s["q_w"], angle, d, False)
        k = _turn64(s["k"][a:a + t], s["k_w"], angle, d, False)
        r = slice(int(s["cu_host"][doc]), int(s["cu_host"][doc]) + length)
        k = torch.cat((kc[r], k)).permute(1, 2, 0).contiguous()
        v = torch.cat((vc[r], s["v"][a:a + t].double()))
        v = v.transpose(0, 1).contiguous()              # [hk, keys, d]
        q = q.view(t, hk, hq // hk, d).transpose(0, 1).reshape(hk, -1, d)
        x = torch.matmul(q, k) / math.sqrt(d)
        x = x.view(hk, t, hq // hk, length + t)
        x[..., length:] += torch.full((t, t), -math.inf, device=DEV,
                                      dtype=x.dtype).triu(1).unsqueeze(1)
        w = torch.softmax(x, -1).view(hk, -1, length + t)
        o = torch.matmul(w, v).view(hk, t, hq // hk, d).transpose(0, 1)
        out[a:a + t] = o.reshape(t, hq, d)
    return out


# ---------------------------------------------------------------------------

def _mean(least, most):
    return (least + most) / 2 if least else most


def work(case):
    """Bytes and operations one pass cannot do without: inputs read and
    outputs written once, prefix states in their 17 bytes a block."""
    h, d = case["kv_heads"], case["head_dim"]
    if case["kind"] == "put":
        e = SIZE[case["dtype"]]
        values = case["docs"] * _mean(case["least"], case["slots"]) * h * d
        return {"bytes": 2 * values * (e + 2), "flops": 2 * values * 10}
    hq = case["q_heads"]
    t = _mean(case["least_tokens"], case["tokens"])
    n = _mean(case["least_slots"], case["slots"])
    total = case["pairs"] * t
    moved = 4 * total * (hq + h) * d + case["docs"] * n * h * d * 2 * 17 / 32
    flops = 4 * hq * d * case["pairs"] * t * (n + (t + 1) / 2)
    return {"bytes": moved, "flops": flops}
