"""Plain 64-bit forms of the operators around the attention, and the bounds
their fp32 kernels are held to (torch, any device)."""
import torch

F64 = torch.float64
# unit roundoff (2^-p for p significant bits) and smallest subnormal step of
# the output types
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11,
        torch.float32: 2.0 ** -24}
STEP = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24,
        torch.float32: 2.0 ** -149}
# fp32 work in front of an output's own rounding, relative to the magnitudes
# that are added: a row sum of up to 65,536 squares has at most 64 terms in
# one lane and 10 levels above it, 74 * 2^-24 < 2^-17; the root halves that,
# division, gains, scales and exponentials of arguments up to 20 (relative
# error 20 log2(e) 2^-24) add less than 2^-18 each.
FP32 = 2.0 ** -15


def norm(v, gain, eps):
    v = v.to(F64)
    if gain is None:
        return v
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * gain.to(F64)


def silu_up(x, up):
    x = x.to(F64)
    return x / (1 + torch.exp(-x)) * up.to(F64)


def product(x, x_scale, w, w_scale, bias=None, residual=None):
    """(y, sum of the magnitudes that are added)."""
    acc = x.to(F64) @ w.to(F64).t().contiguous()
    y = acc * x_scale.to(F64)[:, None] * w_scale.to(F64)[None, :]
    mag = y.abs()
    for t in (bias, residual):
        if t is not None:
            y = y + t.to(F64)
            mag = mag + t.to(F64).abs()
    return y, mag


def rotary(x, positions, inv_freq, interleaved=False, inverse=False,
           factor=1.0, gain=None, eps=1e-6):
    v = norm(x, gain, eps) if gain is not None else x.to(F64)
    half = inv_freq.numel()
    t = positions.to(F64)[:, None] * inv_freq.to(F64)[None, :]
    if inverse:
        t = -t
    c, s = factor * torch.cos(t)[:, None], factor * torch.sin(t)[:, None]
    out = v.clone()
    mag = v.abs().clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        ca, sa = c[..., i], s[..., i]
        out[..., a] = v[..., a] * ca - v[..., b] * sa
        out[..., b] = v[..., b] * ca + v[..., a] * sa
        mag[..., a] = mag[..., b] = abs(factor) * (v[..., a].abs() +
                                                   v[..., b].abs())
    return out, mag


def assert_close(got, ref, mag=None, fp32=FP32):
    """|got - ref| <= the output's rounding + fp32 * mag, elementwise."""
    mag = ref.abs() if mag is None else mag
    err = (got.to(F64) - ref).abs()
    # the rounding is of a value that is itself off by the fp32 bound
    bound = fp32 * mag + UNIT[got.dtype] * (ref.abs() + fp32 * mag) + \
        STEP[got.dtype]
    bad = ~(err <= bound)
    assert not bad.any(), (
        f"{int(bad.sum())} of {bad.numel()} outside the bound, worst "
        f"{(err - bound).max().item():.3e} over it at error "
        f"{err.max().item():.3e}")


def assert_int8_rows(q, scale, v, fp32=FP32):
    """q * scale is v to half a step of the row's largest magnitude at 127."""
    a = v.abs().amax(1).clamp_min(127 * 2.0 ** -126)
    step = a / 127
    assert ((scale.to(F64) - step).abs() <= fp32 * step).all()
    assert (q.to(torch.int32).abs() <= 127).all()
    err = (q.to(F64) * scale.to(F64)[:, None] - v).abs()
    assert (err <= (0.5 + 2 * 127 * fp32) * step[:, None]).all()
