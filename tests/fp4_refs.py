"""Plain forms of the 4-bit prefix store, in 64 bits on the CPU: what a store
holds of given states, and keys normed and turned to their positions."""
import numpy as np
import torch

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def hold(blocks):
    """Values [..., 32] (float64, bf16 values) as their blocks hold them."""
    blocks = np.asarray(blocks, np.float64)
    top = np.abs(blocks).max(-1, keepdims=True)
    fine = np.isfinite(blocks).all(-1, keepdims=True)
    m, x = np.frexp(np.where(fine, top, 1.0))         # top = m 2^x, m < 1
    # 7 * 2^e = 0.875 * 2^(e + 3)
    e = np.where(m <= 0.875, x - 3, x - 2)
    e = np.clip(np.where(top > 0, e, -125), -125, 125)
    unit = np.ldexp(1.0, e)
    t = np.abs(np.where(fine, blocks, 0.0)) / unit
    # the nearest level, ties to the even code
    gap = np.abs(t[..., None] - LEVELS)
    best = gap.min(-1, keepdims=True)
    even = np.arange(8) % 2 == 0
    code = np.argmin(np.where(gap == best, np.where(even, 0, 1), 2), -1)
    out = np.copysign(LEVELS[code] * unit, blocks)
    return np.where(fine, out, np.nan)


def hold_keys(k):
    """k [slots, Hkv, D] float64 -> what a 4-bit store holds."""
    out = np.empty(k.shape)
    for j in range(k.shape[-1] // 64):
        for h in range(2):
            dims = [64 * j + 16 * i + 8 * h + e
                    for i in range(4) for e in range(8)]
            out[..., dims] = hold(k[..., dims])
    return out


def hold_values(v, cu):
    out = np.empty(v.shape)
    for a, b in zip(cu[:-1], cu[1:]):
        for s in range(a, b, 32):
            n = min(32, b - s)
            block = np.zeros((32,) + v.shape[1:])
            block[:n] = v[s:s + n]
            out[s:s + n] = np.moveaxis(hold(np.moveaxis(block, 0, -1)), -1,
                                       0)[:n]
    return out


def held(k, v, cu):
    """bf16 torch tensors [slots, Hkv, D] -> the bf16 tensors a 4-bit store
    reads back as (every held value is a bf16 value)."""
    cu = [int(c) for c in cu]
    hk = torch.from_numpy(hold_keys(k.double().cpu().numpy()))
    hv = torch.from_numpy(hold_values(v.double().cpu().numpy(), cu))
    return hk.to(torch.bfloat16), hv.to(torch.bfloat16)


def turned_keys(k, positions, inv_freq, *, gain=None, interleaved=False,
                factor=1.0, eps=1e-6):
    """k [rows, Hkv, D] (CPU) normed and turned in 64 bits, rounded to fp32
    and from there to bf16."""
    x = k.double()
    if gain is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
        x = x * gain.double()
    r = 2 * inv_freq.numel()
    t = positions.double()[:, None, None] * inv_freq.double()
    c, s = t.cos() * factor, t.sin() * factor
    i = torch.arange(r // 2)
    one = 2 * i if interleaved else i
    two = 2 * i + 1 if interleaved else i + r // 2
    a, b = x[..., one], x[..., two]
    out = x.clone()
    out[..., one], out[..., two] = a * c - b * s, b * c + a * s
    return out.float().to(torch.bfloat16)
