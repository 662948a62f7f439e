"""The operators of a decoder layer around its attention, as measurable cases.

Four operators: the 8-bit integer product with a scale per token and per
channel (``dopr_quant_matmul``), the quantisation of rows that feeds it
(``dopr_quantize_rows``), the norms on either side of a block's gated, scaled
residual (``dopr_norm_residual``), and rotary positions
(``dopr_rotary``).  The shapes are those of the repository's own layers
(Qwen3-0.6B-, 4B- and 8B-shaped), its batches (one pair of 129 online tokens,
one query's 100 candidates, documents of 2048 tokens) and odd ones.

``run`` computes a case with elementary torch operations in 32 bits, or, with
``own`` set, through the library's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
TINY = 127.0 * 2.0 ** -126        # least row maximum that sets a scale

# (outputs, depth) of the layers' products: q, k and v side by side, the
# attention's output, gate and up side by side, down
WIDTHS = {"0p6b": (1024, 2048, 4096, 3072), "4b": (2560, 4096, 6144, 9728),
          "8b": (4096, 4096, 6144, 12288)}


def _projections(width):
    hidden, att, qkv, inter = WIDTHS[width]
    return [(qkv, hidden), (hidden, att), (2 * inter, hidden),
            (hidden, inter)]


def _product(name, rows, cols, depth, dtype="bf16", pitch=16, bias=False,
             residual=False):
    return {"name": name, "kind": "product", "rows": rows, "cols": cols,
            "depth": depth, "dtype": dtype, "pitch": pitch, "bias": bias,
            "residual": residual}


def _linear(name, source, rows, cols, depth, dtype="bf16", residual=False):
    return {"name": name, "kind": "linear", "source": source, "rows": rows,
            "cols": cols, "depth": depth, "dtype": dtype,
            "residual": residual}


def _norm(name, rows, width, dtype="bf16", stream="same", post=False,
          gate="none", pre=True, residual_scale=1.0):
    return {"name": name, "kind": "norm", "rows": rows, "width": width,
            "dtype": dtype, "stream": stream, "post": post, "gate": gate,
            "pre": pre, "residual_scale": residual_scale}


def _rotary(name, sequences, tokens, first, heads, head_dim, rotated,
            dtype="bf16", interleaved=False, norm=False, fused=False,
            factor=1.0, theta=1e6, inverse=False):
    return {"name": name, "kind": "rotary", "sequences": sequences,
            "tokens": tokens, "first": first, "q_heads": heads[0],
            "kv_heads": heads[1], "head_dim": head_dim, "rotated": rotated,
            "dtype": dtype, "interleaved": interleaved, "norm": norm,
            "fused": fused, "factor": factor, "theta": theta,
            "inverse": inverse}


def listed():
    return [
        # q, k and v of one token entering an 8B layer: the weights' bytes
        # and the latency of a call
        _product("product_one_token", 1, 6144, 4096),
        # gate and up of one pair's 129 online tokens, 8B layer
        _product("product_one_pair", 129, 24576, 4096),
        # gate and up of 100 pairs of 32 tokens, 0.6B layer
        _product("product_passages", 3200, 6144, 1024),
        # gate and up of one query's 100 candidates, 8B layer: the largest
        _product("product_one_query", 12900, 24576, 4096),
        # nothing a multiple of anything: rows of odd length, back to back
        _product("product_odd", 1021, 2563, 2501, dtype="f32", pitch=1,
                 bias=True, residual=True),
        # down of a few tokens, 8B layer: SiLU(gate) up in 8 bits, product,
        # residual
        _linear("linear_down_few", "swiglu", 16, 4096, 12288, residual=True),
        # a block's output joins the residual, is normed, goes to 8 bits and
        # through q, k and v of a 4B layer: a ragged batch of some 250 pairs
        _linear("linear_qkv", "norm", 9001, 6144, 2560),
        # both norms around a gated, scaled residual for one query's score
        # tokens
        _norm("norm_score_tokens", 100, 4096, post=True, gate="channel",
              residual_scale=0.7),
        # the plain join of one query's tokens: residual sum and next norm
        _norm("norm_one_query", 12900, 4096),
        # odd width, the residual kept in 32 bits, a gate per token and
        # channel, both norms
        _norm("norm_odd", 20011, 2561, dtype="f16", stream="f32", post=True,
              gate="row", residual_scale=0.5),
        # heads' norm and rotation of one pair's tokens behind a document's
        # 256 prefix slots
        _rotary("rotary_one_pair", 1, 129, 256, (32, 8), 128, 128,
                norm=True),
        # 16 documents of 2048 tokens out of one q, k, v buffer, half of
        # each head rotated in the interleaved layout, scaled for a longer
        # context
        _rotary("rotary_documents", 16, 2048, 0, (32, 8), 128, 64,
                interleaved=True, fused=True, factor=4.0),
    ]


MOST = 12900 * 24576 * 4096       # the largest product's multiplications


def _log_int(rng, lo, hi):
    if hi <= lo:
        return lo
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_product_sizes(rng):
    if rng.random() < 0.6:
        cols, depth = rng.choice(_projections(rng.choice(sorted(WIDTHS))))
    else:
        cols, depth = _log_int(rng, 64, 24576), _log_int(rng, 64, 12288)
    rows = _log_int(rng, 1, min(12900, MOST // (cols * depth)))
    return rows, cols, depth


def draw(rng):
    kind = rng.choices(["product", "linear", "norm", "rotary"],
                       [35, 25, 20, 20])[0]
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "product":
        rows, cols, depth = _draw_product_sizes(rng)
        case = _product("", rows, cols, depth, dtype,
                        rng.choice([16, 16, 16, 1]), rng.random() < 0.3,
                        rng.random() < 0.4)
    elif kind == "linear":
        rows, cols, depth = _draw_product_sizes(rng)
        case = _linear("", rng.choice(["rows", "swiglu", "norm"]), rows, cols,
                       depth, dtype, rng.random() < 0.4)
    elif kind == "norm":
        width = rng.choice([1024, 2560, 4096, _log_int(rng, 64, 12288),
                            _log_int(rng, 64, 12288)])
        rows = _log_int(rng, 1, 20011 * 2561 // width)
        post = rng.random() < 0.5
        case = _norm("", rows, width, dtype, rng.choice(["same", "f32"]),
                     post, rng.choice(["none", "channel", "row"]),
                     not post or rng.random() < 0.7,
                     rng.choice([1.0, rng.uniform(0.2, 1.5)]))
    else:
        head_dim = rng.choice([64, 96, 128, 128, 256])
        rotated = rng.choice([head_dim, head_dim, head_dim // 2,
                              2 * rng.randint(1, head_dim // 2)])
        kv = rng.choice([1, 2, 4, 8, 8])
        heads = (kv * rng.choice([1, 2, 4, 8]), kv)
        most = 32768 * 40 * 128 // ((heads[0] + heads[1]) * head_dim)
        total = _log_int(rng, 1, min(32768, most))
        tokens = _log_int(rng, 1, min(total, 4096))
        inverse = rng.random() < 0.2
        case = _rotary("", max(1, total // tokens), tokens,
                       rng.choice([0, rng.randint(0, 512)]), heads, head_dim,
                       rotated, dtype if dtype != "f32" else "bf16",
                       rng.random() < 0.5,
                       not inverse and rng.random() < 0.5,
                       rng.random() < 0.5, rng.choice([1.0, 2.0, 4.0, 8.0]),
                       rng.choice([1e4, 5e5, 1e6]), inverse)
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# Inputs

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def _activations(gen, rows, width):
    """Hidden states: normal, with a few channels that run much larger."""
    big = torch.rand(width, generator=gen, device=DEV) < 0.004
    return _randn(gen, rows, width) * torch.where(big, 12.0, 1.0)


def _gains(gen, width, dtype):
    return (1.0 + 0.1 * _randn(gen, width)).to(dtype)


def _pitched(values, pitch):
    """`values` with rows a multiple of `pitch` elements apart."""
    rows, width = values.shape
    if width % pitch == 0:
        return values
    wide = -(-width // pitch) * pitch
    buf = torch.zeros(rows, wide, dtype=values.dtype, device=DEV)
    buf[:, :width] = values
    return buf[:, :width]


def _to_int8(v):
    """Rows in 8 bits, each with its largest magnitude at 127."""
    a = v.abs().amax(1).clamp_min(TINY)
    return torch.round(v * (127.0 / a)[:, None]).to(torch.int8), a / 127.0


def _weights(gen, cols, depth, pitch):
    w, scale = _to_int8(_randn(gen, cols, depth) * depth ** -0.5)
    return _pitched(w, pitch), scale


def _empty(*shape, dtype):
    return torch.empty(shape, dtype=dtype, device=DEV)


def _int8_rows(rows, depth):
    """A buffer for quantised rows, on a pitch of 16 bytes."""
    return _empty(rows, -(-depth // 16) * 16, dtype=torch.int8)[:, :depth]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt = TYPES[case["dtype"]]
    s = dict(case)
    if case["kind"] in ("product", "linear"):
        rows, cols, depth = case["rows"], case["cols"], case["depth"]
        pitch = case.get("pitch", 16)
        s["w"], s["w_scale"] = _weights(gen, cols, depth, pitch)
        s["y"] = _empty(rows, cols, dtype=dt)
        s["add"] = (_randn(gen, rows, cols).to(dt) if case["residual"]
                    else None)
        s["bias_v"] = (_randn(gen, cols).to(dt) if case.get("bias")
                       else None)
        if case["kind"] == "product":
            x, s["x_scale"] = _to_int8(_activations(gen, rows, depth))
            s["x"] = _pitched(x, pitch)
        else:
            s["q"] = _int8_rows(rows, depth)
            s["q_scale"] = _empty(rows, dtype=torch.float32)
            if case["source"] == "swiglu":
                s["x"] = _randn(gen, rows, 2 * depth).to(dt)
            else:
                s["x"] = _activations(gen, rows, depth).to(dt)
            if case["source"] == "norm":
                s["stream_in"] = _activations(gen, rows, depth).to(dt)
                s["pre_w"] = _gains(gen, depth, dt)
                s["h"] = _empty(rows, depth, dtype=dt)
        s["workspace"] = None
        if own:
            from paper_2609_03311_amd import dopr_quant_matmul_workspace
            need = dopr_quant_matmul_workspace(rows, cols, depth)
            if need:
                s["workspace"] = _empty(need, dtype=torch.uint8)
    elif case["kind"] == "norm":
        rows, width = case["rows"], case["width"]
        st = dt if case["stream"] == "same" else torch.float32
        s["x"] = _randn(gen, rows, width).to(dt)
        s["stream_in"] = _activations(gen, rows, width).to(st)
        s["post_w"] = _gains(gen, width, dt) if case["post"] else None
        s["pre_w"] = _gains(gen, width, dt) if case["pre"] else None
        shape = {"none": None, "channel": (width,), "row": (rows, width)}
        shape = shape[case["gate"]]
        s["gate_v"] = (None if shape is None else
                       (0.5 * _randn(gen, *shape)).to(dt))
        s["h"] = _empty(rows, width, dtype=st)
        s["z"] = _empty(rows, width, dtype=dt) if case["pre"] else None
    else:
        hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
        n, t = case["sequences"], case["tokens"]
        rows = n * t
        if case["fused"]:
            buf = _randn(gen, rows, (hq + 2 * hk) * d).to(dt)
            s["q"] = buf[:, :hq * d].view(rows, hq, d)
            s["k"] = buf[:, hq * d:(hq + hk) * d].view(rows, hk, d)
        else:
            s["q"] = _randn(gen, rows, hq, d).to(dt)
            s["k"] = _randn(gen, rows, hk, d).to(dt)
        s["q_out"] = _empty(rows, hq, d, dtype=dt)
        s["k_out"] = _empty(rows, hk, d, dtype=dt)
        s["q_w"] = _gains(gen, d, dt) if case["norm"] else None
        s["k_w"] = _gains(gen, d, dt) if case["norm"] else None
        # each sequence starts up to 64 positions behind `first`
        start = case["first"] + torch.randint(0, 65, (n, 1), generator=gen,
                                              device=DEV)
        pos = start + torch.arange(t, device=DEV)[None, :]
        s["positions"] = pos.reshape(-1).to(torch.int32)
        s["inv_freq"], s["mscale"] = _frequencies(case)
    return s


def _frequencies(case):
    """Rotation frequencies of a context `factor` times the trained one
    (4096): wavelengths beyond it stretched, short ones kept, a ramp
    between."""
    r, f = case["rotated"], case["factor"]
    i = torch.arange(0, r, 2, dtype=torch.float64)
    freq = case["theta"] ** (-i / r)
    if f > 1.0:
        turns = 4096 * freq / (2 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        freq = freq * (keep + (1.0 - keep) / f)
    mscale = 1.0 if f <= 1.0 else 0.1 * math.log(f) + 1.0
    return freq.float().to(DEV), mscale


# ---------------------------------------------------------------------------
# One pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2609_03311_amd as D
    if s["kind"] == "product":
        D.dopr_quant_matmul(s["x"], s["x_scale"], s["w"], s["w_scale"],
                            s["y"], bias=s["bias_v"], residual=s["add"],
                            workspace=s["workspace"])
        return s["y"]
    if s["kind"] == "linear":
        if s["source"] == "norm":
            D.dopr_norm_residual(s["x"], residual=s["stream_in"],
                                 pre_norm_w=s["pre_w"], h=s["h"], q=s["q"],
                                 q_scale=s["q_scale"], rms_eps=EPS)
        elif s["source"] == "swiglu":
            k = s["depth"]
            D.dopr_quantize_rows(s["x"][:, :k], s["q"], s["q_scale"],
                                 up=s["x"][:, k:])
        else:
            D.dopr_quantize_rows(s["x"], s["q"], s["q_scale"])
        D.dopr_quant_matmul(s["q"], s["q_scale"], s["w"], s["w_scale"],
                            s["y"], residual=s["add"],
                            workspace=s["workspace"])
        return (s["h"], s["y"]) if s["source"] == "norm" else s["y"]
    if s["kind"] == "norm":
        D.dopr_norm_residual(s["x"], residual=s["stream_in"],
                             post_norm_w=s["post_w"], gate=s["gate_v"],
                             residual_scale=s["residual_scale"],
                             pre_norm_w=s["pre_w"], h=s["h"], z=s["z"],
                             rms_eps=EPS)
        return s["h"] if s["z"] is None else (s["h"], s["z"])
    D.dopr_rotary(s["q"], s["k"], s["positions"], s["inv_freq"], s["q_out"],
                  s["k_out"], interleaved=s["interleaved"],
                  inverse=s["inverse"], attention_factor=s["mscale"],
                  q_norm_w=s["q_w"], k_norm_w=s["k_w"], rms_eps=EPS)
    return s["q_out"], s["k_out"]


def _rms_norm(v, gain):
    inv = 1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * inv * gain.to(v.dtype)


def _scaled_product(x, x_scale, w, w_scale, s):
    y = x.float() @ w.float().t()
    y = y * x_scale[:, None] * w_scale[None, :]
    if s["bias_v"] is not None:
        y = y + s["bias_v"].float()
    if s["add"] is not None:
        y = y + s["add"].float()
    return y.to(s["y"].dtype)


def _rotate(v, gain, s):
    v = v.float()
    if gain is not None:
        v = _rms_norm(v, gain)
    r = s["rotated"]
    angle = s["positions"].float()[:, None] * s["inv_freq"][None, :]
    cos = (torch.cos(angle) * s["mscale"])[:, None, :]
    sin = (torch.sin(angle) * s["mscale"])[:, None, :]
    if s["inverse"]:
        sin = -sin
    if s["interleaved"]:
        a, b = v[..., 0:r:2], v[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin),
                             -1).flatten(-2)
    else:
        a, b = v[..., :r // 2], v[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, v[..., r:]), -1).to(s["q_out"].dtype)


def _run_plain(s):
    if s["kind"] == "product":
        return _scaled_product(s["x"], s["x_scale"], s["w"], s["w_scale"], s)
    if s["kind"] == "linear":
        v = s["x"].float()
        h = None
        if s["source"] == "norm":
            h = v + s["stream_in"].float()
            v = _rms_norm(h, s["pre_w"])
        elif s["source"] == "swiglu":
            g, u = v[:, :s["depth"]], v[:, s["depth"]:]
            v = g / (1.0 + torch.exp(-g)) * u
        q, scale = _to_int8(v)
        y = _scaled_product(q, scale, s["w"], s["w_scale"], s)
        return y if h is None else (h.to(s["h"].dtype), y)
    if s["kind"] == "norm":
        n = s["x"].float()
        if s["post_w"] is not None:
            n = _rms_norm(n, s["post_w"])
        if s["gate_v"] is not None:
            n = n * s["gate_v"].float()
        h = s["residual_scale"] * s["stream_in"].float() + n
        if s["pre_w"] is None:
            return h.to(s["h"].dtype)
        return h.to(s["h"].dtype), _rms_norm(h, s["pre_w"]).to(s["z"].dtype)
    return _rotate(s["q"], s["q_w"], s), _rotate(s["k"], s["k_w"], s)


# ---------------------------------------------------------------------------
# The definition in 64 bits, written apart from the plain form

def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64

    def norm(t, gain):
        power = t.square().sum(-1, keepdim=True) / t.shape[-1]
        return t * torch.rsqrt(power + EPS) * gain.to(f64)

    if case["kind"] in ("product", "linear"):
        h = None
        if case["kind"] == "product":
            left = s["x"].to(f64) * s["x_scale"].to(f64).unsqueeze(1)
        else:
            v = s["x"].to(f64)
            if case["source"] == "norm":
                h = v + s["stream_in"].to(f64)
                v = norm(h, s["pre_w"])
            elif case["source"] == "swiglu":
                g, u = v.split(case["depth"], dim=1)
                v = g * torch.sigmoid(g) * u
            step = v.abs().max(dim=1, keepdim=True).values / 127.0
            step = torch.where(step > 0, step, torch.ones_like(step))
            left = torch.round(v / step) * step
        right = s["w"].to(f64) * s["w_scale"].to(f64).unsqueeze(1)
        y = torch.matmul(left, right.t().contiguous())
        if s["bias_v"] is not None:
            y += s["bias_v"].to(f64)
        if s["add"] is not None:
            y += s["add"].to(f64)
        return y if h is None else (h, y)
    if case["kind"] == "norm":
        n = s["x"].to(f64)
        if case["post"]:
            n = norm(n, s["post_w"])
        if case["gate"] != "none":
            n = n * s["gate_v"].to(f64)
        h = n + case["residual_scale"] * s["stream_in"].to(f64)
        return (h, norm(h, s["pre_w"])) if case["pre"] else h

    # rotation as the product of complex numbers, pair by pair
    def turn(t, gain):
        t = t.to(f64)
        if gain is not None:
            t = norm(t, gain)
        half = case["rotated"] // 2
        i = torch.arange(half, device=t.device)
        first = 2 * i if case["interleaved"] else i
        second = first + (1 if case["interleaved"] else half)
        angle = s["positions"].to(f64).unsqueeze(1) * s["inv_freq"].to(f64)
        if case["inverse"]:
            angle = -angle
        unit = torch.polar(torch.full_like(angle, s["mscale"]), angle)
        z = torch.complex(t[..., first], t[..., second]) * unit.unsqueeze(1)
        out = t.clone()
        out[..., first] = z.real
        out[..., second] = z.imag
        return out

    return turn(s["q"], s["q_w"]), turn(s["k"], s["k_w"])


# ---------------------------------------------------------------------------

def work(case):
    """Bytes and operations one pass cannot do without: inputs read and
    outputs written once."""
    e = SIZE[case["dtype"]]
    if case["kind"] in ("product", "linear"):
        m, n, k = case["rows"], case["cols"], case["depth"]
        moved = n * k + 4 * n + m * n * e * (2 if case["residual"] else 1)
        flops = 2 * m * n * k
        if case["kind"] == "product":
            moved += m * k + 4 * m + (n * e if case["bias"] else 0)
        elif case["source"] == "rows":
            moved += m * k * e
            flops += 3 * m * k
        elif case["source"] == "swiglu":
            moved += 2 * m * k * e
            flops += 8 * m * k
        else:
            moved += 3 * m * k * e + k * e
            flops += 8 * m * k
        return {"bytes": moved, "flops": flops}
    if case["kind"] == "norm":
        m, w = case["rows"], case["width"]
        es = e if case["stream"] == "same" else 4
        moved = m * w * (e + 2 * es)
        moved += w * e * (int(case["post"]) + int(case["pre"]))
        moved += m * w * e if case["pre"] else 0
        moved += {"none": 0, "channel": w * e, "row": m * w * e}[case["gate"]]
        return {"bytes": moved, "flops": 12 * m * w}
    rows = case["sequences"] * case["tokens"]
    heads = case["q_heads"] + case["kv_heads"]
    values = rows * heads * case["head_dim"]
    return {"bytes": 2 * values * e + 4 * rows + 2 * case["rotated"],
            "flops": values * (6 + (4 if case["norm"] else 0))}
