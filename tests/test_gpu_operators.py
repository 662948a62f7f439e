"""The operators around the attention against their plain 64-bit forms (GPU):
8-bit integer rows and products, norms around a gated residual, rotary
positions.  The bounds are derived in operator_refs.py."""
import gc

import numpy as np
import pytest
import torch

import operator_refs as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
GUARD = -77.0


def _D():
    import paper_2609_03311_amd as D
    return D


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (scale * torch.randn(shape, generator=g, device=DEV)).to(dtype)


class Guarded:
    """A [rows, width] view with `gap` elements between rows, at an element
    offset, in a buffer whose other elements must stay as they are."""

    def __init__(self, rows, width, dtype, gap=0, offset=0):
        pitch = width + gap
        mark = GUARD if dtype.is_floating_point else -77
        self.mark = mark
        self.buf = torch.full((offset + rows * pitch + 64,), mark,
                              dtype=dtype, device=DEV)
        self.view = torch.as_strided(self.buf, (rows, width), (pitch, 1),
                                     offset)

    def set(self, values):
        self.view.copy_(values)
        return self.view

    def check(self):
        """Every element outside the view still holds the mark."""
        own = torch.zeros_like(self.buf, dtype=torch.bool)
        torch.as_strided(own, self.view.shape, self.view.stride(),
                         self.view.storage_offset()).fill_(True)
        assert (self.buf[~own] == self.mark).all(), "wrote outside its rows"


# ---------------------------------------------------------------------------
# rows in 8 bits

WIDTHS = [8, 9, 15, 64, 127, 511, 513, 1024, 2048, 2051, 4096, 9728, 12288,
          16390, 40000, 65536]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_quantize_is_the_definition_bit_for_bit(width, dtype):
    """Without `up` every step is one IEEE fp32 operation: equal bits."""
    D = _D()
    g = gen(width)
    rows = 5
    x = Guarded(rows, width, dtype, gap=width % 3, offset=width % 5)
    v = randn(g, rows, width)
    v[1] *= 1e-3
    v[2] = 0                       # a row of zeros
    v[3, width // 2] = 900.0       # one element takes the whole range
    x.set(v.to(dtype))
    q = Guarded(rows, width, torch.int8, gap=width % 7, offset=width % 3)
    s = Guarded(1, rows, torch.float32, offset=1)
    D.dopr_quantize_rows(x.view, q.view, s.view[0])
    f = x.view.float().cpu().numpy()
    a = np.maximum(np.abs(f).max(1), np.float32(127 * 2.0 ** -126))
    scale = a / np.float32(127)
    want = np.rint(f * (np.float32(127) / a)[:, None]).astype(np.int8)
    assert np.array_equal(q.view.cpu().numpy(), want)
    assert np.array_equal(s.view[0].cpu().numpy(), scale)
    for b in (x, q, s):
        b.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(1, 8), (3, 100), (7, 1024),
                                        (2, 3001), (129, 12288), (6, 65535)])
def test_quantize_swiglu(rows, width, dtype):
    D = _D()
    g = gen(rows * width)
    both = randn(g, rows, 2 * width, dtype=dtype, scale=2.0)
    x, up = both[:, :width], both[:, width:]
    q = torch.empty(rows, width, dtype=torch.int8, device=DEV)
    s = torch.empty(rows, device=DEV)
    D.dopr_quantize_rows(x, q, s, up=up)
    R.assert_int8_rows(q, s, R.silu_up(x, up))


@pytest.mark.parametrize("width", [64, 5000])
def test_quantize_rows_that_are_not_finite(width):
    """Such a row has scale NaN and integers 0; its neighbours are as ever.
    Tiny rows keep a normal scale."""
    D = _D()
    x = randn(gen(3), 8, width)
    x[1, 3] = float("nan")
    x[2, width - 1] = float("inf")
    x[4, 0] = float("-inf")
    x[5] = 0
    x[5, 1] = 1e-42                # subnormal: below the least maximum
    x[6] = 3.0e38
    q = torch.empty(8, width, dtype=torch.int8, device=DEV)
    s = torch.empty(8, device=DEV)
    D.dopr_quantize_rows(x, q, s)
    bad = [1, 2, 4]
    assert torch.isnan(s[bad]).all() and (q[bad] == 0).all()
    good = [0, 3, 5, 6, 7]
    assert torch.isfinite(s[good]).all() and (s[good] >= 2.0 ** -126).all()
    R.assert_int8_rows(q[good], s[good], x[good].double())
    assert (q[6] == 127).all() and (q[5] == 0).all()
    # SiLU of a large negative times a finite `up` is 0, not NaN
    x = torch.full((1, width), -200.0, device=DEV)
    D.dopr_quantize_rows(x, q[:1], s[:1], up=torch.ones_like(x))
    assert torch.isfinite(s[:1]).all() and (q[:1] == 0).all()


# ---------------------------------------------------------------------------
# products

def int8(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, device=DEV,
                         dtype=torch.int8)


def run_product(m, n, k, dtype, *, x_gap=0, w_gap=0, offset=0, y_gap=0,
                bias=False, residual=False, in_place=False, seed=0):
    D = _D()
    g = gen(seed + m + n + k)
    x = Guarded(m, k, torch.int8, gap=x_gap, offset=offset)
    w = Guarded(n, k, torch.int8, gap=w_gap, offset=offset)
    x.set(int8(g, m, k))
    w.set(int8(g, n, k))
    xs = torch.rand(m, generator=g, device=DEV) / 127
    ws = torch.rand(n, generator=g, device=DEV) / 127 / max(k, 1) ** 0.5
    b = randn(g, n, dtype=dtype) if bias else None
    y = Guarded(m, n, dtype, gap=y_gap, offset=offset)
    r = None
    if residual:
        vals = randn(g, m, n, dtype=dtype)
        r = y.set(vals) if in_place else vals
    ref, mag = R.product(x.view, xs, w.view, ws, b, r)
    need = D.dopr_quant_matmul_workspace(m, n, k)
    # (the workspace holds what an earlier call left in it)
    wsp = torch.full((max(need, 1),), 0x5a, dtype=torch.uint8, device=DEV)
    wsp = wsp if need else None
    D.dopr_quant_matmul(x.view, xs, w.view, ws, y.view, bias=b, residual=r,
                        workspace=wsp)
    first = y.view.clone()
    R.assert_close(first, ref, mag)
    y.check()
    if not in_place:
        y.view.zero_()
        D.dopr_quant_matmul(x.view, xs, w.view, ws, y.view, bias=b,
                            residual=r, workspace=wsp)
        assert torch.equal(y.view, first), "differs from run to run"


SHAPES = [(1, 1, 1), (1, 16, 16), (1, 4096, 4096), (2, 33, 64), (3, 64, 65),
          (15, 17, 129), (16, 128, 1024), (17, 100, 255), (31, 1000, 640),
          (32, 256, 2560), (33, 130, 96), (48, 2560, 9728), (63, 65, 192),
          (64, 512, 4096), (65, 63, 127), (100, 1024, 2048), (127, 129, 128),
          (128, 128, 128), (129, 6144, 4096), (200, 257, 1000),
          (255, 255, 257), (256, 256, 256), (257, 300, 384), (511, 700, 513),
          (512, 4096, 1024), (777, 1111, 333), (1024, 2560, 4096),
          (2049, 520, 272), (4100, 1030, 528)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_shapes(m, n, k):
    """Rows on 16-byte strides (the bytes behind them hold other values)."""
    run_product(m, n, k, torch.bfloat16, x_gap=-k % 16, w_gap=-k % 16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 70, 100), (16, 256, 512),
                                   (40, 129, 1000), (129, 300, 257),
                                   (300, 513, 1024), (1000, 1500, 400)])
def test_product_bias_residual_types(m, n, k, dtype):
    for i, (bias, res, inp) in enumerate(((True, False, False),
                                          (False, True, False),
                                          (True, True, True))):
        run_product(m, n, k, dtype, x_gap=-k % 16, w_gap=-k % 16,
                    bias=bias, residual=res, in_place=inp, seed=i)


@pytest.mark.parametrize("m,n,k", [(1, 65, 4097), (5, 33, 31), (16, 64, 64),
                                   (70, 129, 1023), (260, 300, 515),
                                   (600, 520, 777)])
def test_product_unaligned(m, n, k):
    """Rows back to back at odd lengths, odd offsets, odd strides."""
    run_product(m, n, k, torch.bfloat16, offset=3)
    run_product(m, n, k, torch.float32, x_gap=5, w_gap=1, y_gap=3, offset=1,
                residual=True)
    run_product(m, n, k, torch.float16, x_gap=16 - k % 16, w_gap=7, y_gap=2,
                bias=True)


@pytest.mark.parametrize("m,n,k", [(17, 33, 129), (70, 129, 1023),
                                   (300, 520, 64), (1021, 515, 2501)])
def test_product_of_rows_laid_out_again(m, n, k):
    """Rows off 16-byte addresses: the same bits with a workspace (laid out
    again), with one too small and without (multiplied as they lie)."""
    D = _D()
    g = gen(m)
    x = Guarded(m, k, torch.int8, gap=1, offset=1)
    w = Guarded(n, k, torch.int8, gap=3, offset=5)
    x.set(int8(g, m, k))
    w.set(int8(g, n, k))
    xs, ws = torch.rand(m, device=DEV), torch.rand(n, device=DEV)
    need = (m + n) * -(-k // 128) * 128
    out = []
    for size in (None, need - 1, need, need + 1000):
        y = Guarded(m, n, torch.float32)
        wsp = None if size is None else torch.full(
            (size,), 0x5a, dtype=torch.uint8, device=DEV)
        D.dopr_quant_matmul(x.view, xs, w.view, ws, y.view, workspace=wsp)
        y.check()
        out.append(y.view)
        if size == need - 1:
            assert (wsp == 0x5a).all()
    R.assert_close(out[0], *R.product(x.view, xs, w.view, ws))
    assert all(torch.equal(o, out[0]) for o in out[1:])


def test_product_empty_depth_and_extremes():
    """Depth 0 leaves bias and residual; -128 and full depth stay exact."""
    D = _D()
    run_product(3, 40, 0, torch.float32, bias=True, residual=True)
    run_product(130, 129, 0, torch.bfloat16, residual=True)
    for m in (1, 40, 129):
        k = 131071
        x = torch.full((m, k + 1), -128, dtype=torch.int8, device=DEV)[:, :k]
        w = torch.full((20, k + 1), -128, dtype=torch.int8, device=DEV)[:, :k]
        w[3] = 127
        one = torch.ones(max(m, 20), device=DEV)
        y = torch.empty(m, 20, device=DEV)
        need = D.dopr_quant_matmul_workspace(m, 20, k)
        wsp = torch.empty(need, dtype=torch.uint8, device=DEV) if need else \
            None
        D.dopr_quant_matmul(x, one[:m], w, one[:20], y, workspace=wsp)
        want = torch.full((20,), 16384.0 * k, dtype=torch.float64)
        want[3] = -128.0 * 127 * k
        assert torch.equal(y.cpu(), want.float().expand(m, 20)), m


def test_product_nan_scale_stays_in_its_row():
    D = _D()
    g = gen(5)
    for m in (4, 60, 300):
        x, w = int8(g, m, 256), int8(g, 80, 256)
        x[2] = 0
        xs = torch.ones(m, device=DEV)
        xs[2] = float("nan")
        y = torch.empty(m, 80, device=DEV)
        need = D.dopr_quant_matmul_workspace(m, 80, 256)
        wsp = torch.empty(need, dtype=torch.uint8, device=DEV) if need else \
            None
        D.dopr_quant_matmul(x, xs, w, torch.ones(80, device=DEV), y,
                            workspace=wsp)
        assert torch.isnan(y[2]).all()
        keep = [i for i in range(m) if i != 2]
        assert torch.isfinite(y[keep]).all()


@pytest.mark.parametrize("m,n", [(3, 40), (40, 3), (130, 140)])
def test_product_offsets_past_32_bits(m, n):
    """Rows so far apart that byte offsets pass 2^31 and 2^32."""
    D = _D()
    g = gen(9)
    k = 272
    far = (5 << 30) // m // 16 * 16
    x = torch.empty(m * far, dtype=torch.int8, device=DEV).as_strided(
        (m, k), (far, 1))
    x.copy_(int8(g, m, k))
    w = int8(g, n, k)
    far_y = (3 << 30) // m // 16 * 16
    y = torch.empty(m * far_y, dtype=torch.bfloat16,
                    device=DEV).as_strided((m, n), (far_y, 1))
    xs, ws = torch.rand(m, device=DEV), torch.rand(n, device=DEV)
    need = D.dopr_quant_matmul_workspace(m, n, k)
    wsp = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    D.dopr_quant_matmul(x, xs, w, ws, y, workspace=wsp)
    R.assert_close(y, *R.product(x, xs, w, ws))
    # the same with w far apart
    farw = (5 << 30) // n // 16 * 16
    wf = torch.empty(n * farw, dtype=torch.int8, device=DEV).as_strided(
        (n, k), (farw, 1))
    wf.copy_(w)
    y2 = torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    D.dopr_quant_matmul(x, xs, wf, ws, y2, workspace=wsp)
    assert torch.equal(y2, y)
    del x, y, wf
    gc.collect()
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------
# norms around a gated residual

def run_norm(rows, width, dtype, stream, *, post, gate, residual, pre, z, q,
             rs=0.75, eps=1e-6, gap=0, offset=0, in_place=False, seed=0,
             scale=1.0):
    D = _D()
    g = gen(seed + rows + width)
    st = dtype if stream == "same" else torch.float32
    x = Guarded(rows, width, dtype, gap=gap, offset=offset)
    x.set(randn(g, rows, width, dtype=dtype, scale=scale))
    pw = (1 + 0.1 * randn(g, width)).to(dtype) if post else None
    nw = (1 + 0.1 * randn(g, width)).to(dtype) if pre else None
    gt = {"none": None, "channel": lambda: randn(g, width, dtype=dtype),
          "row": lambda: randn(g, rows, width, dtype=dtype)}[gate]
    gt = gt() if gt else None
    h = Guarded(rows, width, st, gap=gap, offset=offset)
    r = None
    if residual:
        vals = randn(g, rows, width, dtype=st, scale=scale)
        r = h.set(vals) if in_place else vals
    n = R.norm(x.view, pw, eps)
    gn = n if gt is None else n * gt.double()
    ref_h, mag_h = gn, gn.abs()
    if r is not None:
        ref_h = ref_h + rs * r.double()
        mag_h = mag_h + (rs * r.double()).abs()
    ref_z = R.norm(ref_h, nw, eps)
    # what is off in h is off in z by the same factor
    inv = 1.0
    if pre:
        inv = nw.double().abs() / torch.sqrt(
            (ref_h ** 2).mean(-1, keepdim=True) + eps)
    mag_z = mag_h * inv + ref_z.abs()
    zo = Guarded(rows, width, dtype, gap=gap, offset=offset) if z else None
    qo = Guarded(rows, width, torch.int8, gap=gap, offset=offset) if q else \
        None
    qs = torch.full((rows,), GUARD, device=DEV) if q else None
    D.dopr_norm_residual(x.view, residual=r, post_norm_w=pw, gate=gt,
                         residual_scale=rs, pre_norm_w=nw, h=h.view,
                         z=zo.view if z else None, q=qo.view if q else None,
                         q_scale=qs, rms_eps=eps)
    R.assert_close(h.view, ref_h, mag_h)
    h.check()
    x.check()
    if z:
        R.assert_close(zo.view, ref_z, mag_z)
        zo.check()
    if q:
        # a value is off by the fp32 bound of its terms before it is rounded
        amax = ref_z.abs().amax(1)
        ratio = (mag_z.amax(1) / amax.clamp_min(1e-300)).max().item()
        R.assert_int8_rows(qo.view, qs, ref_z, R.FP32 * max(ratio, 1.0))
        qo.check()


@pytest.mark.parametrize("width", [8, 11, 64, 500, 1024, 2048, 2561, 4096,
                                   8200, 12288, 20000, 65536])
def test_norm_widths(width):
    run_norm(6, width, torch.bfloat16, "same", post=True, gate="channel",
             residual=True, pre=True, z=True, q=True)
    run_norm(1, width, torch.float16, "f32", post=False, gate="none",
             residual=True, pre=True, z=False, q=True, gap=3, offset=1)


@pytest.mark.parametrize("dtype,stream", [(torch.bfloat16, "same"),
                                          (torch.bfloat16, "f32"),
                                          (torch.float16, "same"),
                                          (torch.float16, "f32"),
                                          (torch.float32, "same")])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("gate", ["none", "channel", "row"])
def test_norm_forms(dtype, stream, post, pre, gate):
    for i, residual in enumerate((False, True)):
        run_norm(37, 1030, dtype, stream, post=post, gate=gate,
                 residual=residual, pre=pre, z=True, q=bool(i), gap=2 * i,
                 offset=i, in_place=residual, seed=i)


def test_norm_zero_rows_and_large_values():
    """A row of zeros gives zeros; rows near the type's ends stay finite."""
    D = _D()
    for width in (64, 5000):
        x = torch.zeros(3, width, dtype=torch.bfloat16, device=DEV)
        x[1] = 2.0 ** 60
        x[2] = 2.0 ** -60
        w = torch.ones(width, dtype=torch.bfloat16, device=DEV)
        z = torch.empty_like(x)
        q = torch.empty(3, width, dtype=torch.int8, device=DEV)
        s = torch.empty(3, device=DEV)
        D.dopr_norm_residual(x, pre_norm_w=w, z=z, q=q, q_scale=s)
        assert (z[0] == 0).all() and (q[0] == 0).all()
        assert (z[1] == 1).all() and (q[1] == 127).all()
        R.assert_close(z, R.norm(x, w, 1e-6))
        x[1, 5] = float("nan")
        D.dopr_norm_residual(x, pre_norm_w=w, z=z, q=q, q_scale=s)
        assert torch.isnan(z[1]).all() and torch.isnan(s[1])
        assert (q[1] == 0).all()
        assert torch.isfinite(z[[0, 2]].float()).all()


def test_norm_in_place_in_every_operand():
    """h over the residual and z over x at once: the same bits as apart."""
    D = _D()
    for width in (40, 1027, 4096, 9001):
        g = gen(width)
        x = randn(g, 19, width, dtype=torch.bfloat16)
        r = randn(g, 19, width, dtype=torch.bfloat16)
        w = randn(g, width, dtype=torch.bfloat16)
        h, z = torch.empty_like(x), torch.empty_like(x)
        kw = dict(post_norm_w=w, pre_norm_w=w, residual_scale=0.5)
        D.dopr_norm_residual(x, residual=r, h=h, z=z, **kw)
        D.dopr_norm_residual(x, residual=r, h=r, z=x, **kw)
        assert torch.equal(h, r) and torch.equal(z, x)


# ---------------------------------------------------------------------------
# rotary positions

def run_rotary(rows, hq, hk, d, r, dtype, *, interleaved=False, inverse=False,
               normed=False, factor=1.0, fused=False, heads_first=False,
               in_place=False, top=5000, seed=0):
    D = _D()
    g = gen(seed + rows + d + r)
    if fused:
        buf = randn(g, rows, (hq + 2 * hk) * d + 3, dtype=dtype)
        q = buf[:, 1:1 + hq * d].unflatten(1, (hq, d))
        k = buf[:, 1 + hq * d:1 + (hq + hk) * d].unflatten(1, (hk, d))
    elif heads_first:
        q = randn(g, hq, rows, d, dtype=dtype).transpose(0, 1)
        k = randn(g, hk, rows, d, dtype=dtype).transpose(0, 1)
    else:
        q = randn(g, rows, hq, d, dtype=dtype)
        k = randn(g, rows, hk, d, dtype=dtype)
    pos = torch.randint(0, top, (rows,), generator=g, device=DEV,
                        dtype=torch.int32)
    pos[0] = 0
    freq, _ = D.dopr_rotary_frequencies(r, 1e4)
    freq = freq.to(DEV)
    qw = (1 + 0.1 * randn(g, d)).to(dtype) if normed else None
    kw = (1 + 0.1 * randn(g, d)).to(dtype) if normed else None
    ref = [R.rotary(x, pos, freq, interleaved, inverse, factor, w)
           for x, w in ((q, qw), (k, kw))]
    rest = buf.clone() if fused else None
    qo, ko = (q, k) if in_place else (torch.empty_like(q),
                                      torch.empty_like(k))
    D.dopr_rotary(q, k, pos, freq, qo, ko, interleaved=interleaved,
                  inverse=inverse, attention_factor=factor, q_norm_w=qw,
                  k_norm_w=kw)
    for out, (want, mag) in zip((qo, ko), ref):
        R.assert_close(out, want, mag)
        if r < d and not normed and not in_place:
            src = q if out is qo else k
            assert torch.equal(out[..., r:], src[..., r:])
    if fused and in_place:
        n = 1 + (hq + hk) * d
        assert torch.equal(buf[:, n:], rest[:, n:])
        assert torch.equal(buf[:, 0], rest[:, 0])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,r", [(2, 2), (6, 4), (16, 16), (20, 16), (64, 64),
                                 (64, 32), (64, 10), (80, 80), (96, 96),
                                 (96, 72), (100, 50), (128, 128), (128, 64),
                                 (128, 126), (160, 40), (256, 256), (256, 64),
                                 (512, 512), (512, 34)])
def test_rotary_head_sizes(d, r, interleaved):
    for i, dtype in enumerate(TYPES):
        run_rotary(5, 3, 1, d, r, dtype, interleaved=interleaved,
                   normed=i != 1, factor=1.0 + 0.25 * i, seed=i)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hk", [(1, 1, 1), (1, 32, 8), (129, 32, 8),
                                        (7, 5, 0), (3, 0, 7), (2500, 16, 8),
                                        (40, 130, 3)])
def test_rotary_heads(rows, hq, hk, interleaved):
    kw = dict(interleaved=interleaved, fused=True)
    run_rotary(rows, hq, hk, 128, 128, torch.bfloat16, normed=True, **kw)
    run_rotary(rows, hq, hk, 128, 64, torch.bfloat16, in_place=True, **kw)
    run_rotary(rows, hq, hk, 64, 64, torch.float16, inverse=True,
               heads_first=True, interleaved=interleaved)


def test_rotary_far_positions():
    """Angles of positions up to 2^31 - 1, and negative ones, are reduced in
    64 bits: fp32 outputs stay at fp32 accuracy."""
    D = _D()
    pos = torch.tensor([0, 1, 131072, 1 << 20, (1 << 24) + 1, (1 << 31) - 1,
                        -5, -(1 << 31)], dtype=torch.int32, device=DEV)
    x = randn(gen(1), pos.numel(), 2, 128)
    freq, _ = D.dopr_rotary_frequencies(128, 1e6)
    out = torch.empty_like(x)
    D.dopr_rotary(x, None, pos, freq.to(DEV), out, None)
    # beyond fp32: position * frequency in 64 bits is off by 2^-53 * 2^31
    R.assert_close(out, *R.rotary(x, pos, freq.to(DEV)), fp32=2.0 ** -20)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,r", [(128, 64), (128, 60), (67, 66), (65, 10),
                                 (24, 18), (9, 2)])
def test_rotary_leaves_the_rest_as_it_is(d, r, interleaved):
    """Elements behind the rotated part keep their bits, next to turning ones
    and with infinities among them; the turning ones stay finite."""
    D = _D()
    x = randn(gen(d + r), 7, 3, d)
    x[:, 1, r:] = float("inf")
    x[:, 2, r:] = -0.0
    out = torch.empty_like(x)
    pos = torch.arange(7, device=DEV, dtype=torch.int32)
    freq = D.dopr_rotary_frequencies(r, 1e4)[0].to(DEV)
    D.dopr_rotary(x, None, pos, freq, out, None, interleaved=interleaved)
    assert torch.equal(out[..., r:].view(torch.int32),
                       x[..., r:].view(torch.int32))
    R.assert_close(out[..., :r], *[v[..., :r] for v in R.rotary(
        torch.cat((x[..., :r], torch.zeros_like(x[..., r:])), -1), pos, freq,
        interleaved)])


@pytest.mark.parametrize("dtype", TYPES)
def test_rotary_norm_of_tiny_heads(dtype):
    """Without an epsilon, heads whose mean square is subnormal in fp32 are
    normed like any other."""
    D = _D()
    scale = 2.0 ** -18 if dtype == torch.float16 else 2.0 ** -66
    x = randn(gen(8), 5, 4, 128, dtype=dtype, scale=scale)
    pos = torch.arange(5, device=DEV, dtype=torch.int32)
    freq = D.dopr_rotary_frequencies(128, 1e4)[0].to(DEV)
    w = torch.ones(128, dtype=dtype, device=DEV)
    out = torch.empty_like(x)
    D.dopr_rotary(x, None, pos, freq, out, None, q_norm_w=w, rms_eps=0.0)
    # subnormal squares keep 2^-149 each: 128 of them, of a mean of 2^-132
    R.assert_close(out, *R.rotary(x, pos, freq, gain=w, eps=0.0),
                   fp32=2.0 ** -15 + 2.0 ** -16)


def test_rotary_inverse_undoes_it():
    D = _D()
    x = randn(gen(2), 50, 4, 64)
    pos = torch.arange(50, device=DEV, dtype=torch.int32)
    freq = D.dopr_rotary_frequencies(48, 1e4)[0].to(DEV)
    y, z = torch.empty_like(x), torch.empty_like(x)
    for inter in (False, True):
        D.dopr_rotary(x, None, pos, freq, y, None, interleaved=inter)
        D.dopr_rotary(y, None, pos, freq, z, None, interleaved=inter,
                      inverse=True)
        assert (z - x).abs().max() <= 2.0 ** -20 * x.abs().max()


def test_rotary_offsets_past_32_bits():
    """Heads and tokens whose element offsets pass 2^31."""
    D = _D()
    far = 1 << 30
    x = torch.empty(3 * far + 4096, dtype=torch.bfloat16,
                    device=DEV).as_strided((3, 2, 128), (far, 2048, 1))
    x.copy_(randn(gen(4), 3, 2, 128))
    y = torch.empty(3 * far, dtype=torch.bfloat16,
                    device=DEV).as_strided((2, 3, 128), (128, far, 1)
                                           ).transpose(0, 1)
    pos = torch.tensor([3, 4, 5], device=DEV, dtype=torch.int32)
    freq = D.dopr_rotary_frequencies(128, 1e4)[0].to(DEV)
    D.dopr_rotary(x, None, pos, freq, y, None)
    R.assert_close(y, *R.rotary(x, pos, freq))
    del x, y
    gc.collect()
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------

def test_operators_on_another_stream():
    """Calls run on the stream they are given, in order with its work."""
    D = _D()
    side = torch.cuda.Stream()
    x = torch.zeros(300, 1024, dtype=torch.bfloat16, device=DEV)
    w = int8(gen(1), 64, 1024)
    ws = torch.full((64,), 1e-4, device=DEV)
    q = torch.empty(300, 1024, dtype=torch.int8, device=DEV)
    s = torch.empty(300, device=DEV)
    y = torch.empty(300, 64, dtype=torch.bfloat16, device=DEV)
    need = D.dopr_quant_matmul_workspace(300, 64, 1024)
    wsp = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x.copy_(randn(gen(2), 300, 1024))
    D.dopr_quantize_rows(x, q, s, stream=side)
    D.dopr_quant_matmul(q, s, w, ws, y, stream=side, workspace=wsp)
    side.synchronize()
    R.assert_int8_rows(q, s, x.double())
    R.assert_close(y, *R.product(q, s, w, ws))
