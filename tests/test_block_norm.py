"""sjd_block_norm: refusals without a GPU, values on one against the formula in 64 bits."""
import itertools

import pytest
import torch

from paper_2410_01699_b200 import binding as B

FAKE = 1 << 20   # an address that no refused call may use
E = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _call(**kw):
    a = dict(rows=4, d=64, kind=0, eps=1e-5, dtype=1, h_dtype=1, h=FAKE, hs=64, y=FAKE, ys=64, post_gain=FAKE, post_bias=None, gate=None,
             gate_rows=0, gate_tanh=0, scale=1.0, h_out=FAKE, hos=64, pre_gain=FAKE, pre_bias=None, z=FAKE, zs=64)
    a.update(kw)
    return B.lib().sjd_block_norm(*a.values(), None)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), B.SJD_ERR_BAD_ARG), (dict(d=0), B.SJD_ERR_BAD_ARG), (dict(h=None), B.SJD_ERR_BAD_ARG), (dict(eps=-1.0), B.SJD_ERR_BAD_ARG),
    (dict(eps=float("nan")), B.SJD_ERR_BAD_ARG), (dict(h_out=None), B.SJD_ERR_BAD_ARG), (dict(y=None), B.SJD_ERR_BAD_ARG),
    (dict(y=None, h_out=None), B.SJD_ERR_BAD_ARG), (dict(z=None), B.SJD_ERR_BAD_ARG), (dict(pre_gain=None), B.SJD_ERR_BAD_ARG),
    (dict(y=None, h_out=None, post_gain=None, pre_gain=None, z=None), B.SJD_ERR_BAD_ARG), (dict(post_gain=None, post_bias=FAKE), B.SJD_ERR_BAD_ARG),
    (dict(pre_gain=None, z=None, pre_bias=FAKE), B.SJD_ERR_BAD_ARG), (dict(gate=FAKE), B.SJD_ERR_BAD_ARG), (dict(hs=63), B.SJD_ERR_BAD_ARG),
    (dict(ys=63), B.SJD_ERR_BAD_ARG), (dict(hos=63), B.SJD_ERR_BAD_ARG), (dict(zs=63), B.SJD_ERR_BAD_ARG), (dict(y=FAKE + 1), B.SJD_ERR_BAD_ARG),
    (dict(h_dtype=0, h=FAKE + 2), B.SJD_ERR_BAD_ARG), (dict(dtype=2), B.SJD_ERR_UNSUPPORTED), (dict(h_dtype=-1), B.SJD_ERR_UNSUPPORTED),
    (dict(kind=2), B.SJD_ERR_UNSUPPORTED), (dict(d=32769, hs=32769, ys=32769, hos=32769, zs=32769), B.SJD_ERR_UNSUPPORTED), (dict(rows=0), B.SJD_OK)])
def test_refusals(change, status):
    assert _call(**change) == status


def test_binding_refuses_tensors_of_the_host():
    with pytest.raises(ValueError):
        B.sjd_block_norm(torch.zeros(2, 8), pre_gain=torch.ones(8))


def _norm(x, dx, gain, bias, layer, eps):
    """N(x) gain + bias in 64 bits, and how far fp32 arithmetic may be off where x is by up to dx.  A sum of d entries is at most 32 of a
    thread, 5 levels of a warp and 5 of a block: 42 roundings (E each) of at most the sum of magnitudes; with the quotient, the root and the
    products 64 in all.  Errors of x shift its entry, its mean and its root mean square."""
    mean = x.mean(1, keepdim=True) if layer else 0.0
    c = x - mean
    f = (c.square().mean(1, keepdim=True) + eps).rsqrt()
    g = gain.double().abs()
    n = c * f
    dc = dx + (dx.mean(1, keepdim=True) if layer else 0.0) + (64 * E * x.abs().mean(1, keepdim=True) if layer else 0.0) + E * c.abs()
    off = g * f * dc + (n * gain.double()).abs() * (64 * E + f * dc.square().mean(1, keepdim=True).sqrt())
    out = n * gain.double() + (bias.double() if bias is not None else 0.0)
    return out, off + 2 * E * out.abs()


def _check(rows, d, dtype, h_dtype, kind, post, gates, tanh, pre, biases, scale=1.0, seed=0, offset=0.0, pad=0, eps=1e-5):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    t, ht, layer = DT[dtype], DT[h_dtype], kind == B.SJD_NORM_LAYER
    place = lambda x, dt: torch.cat((x, rnd(x.shape[0], pad)), 1).to(dt).cuda()[:, :d]   # (rows are parts of longer ones)
    h, y = place(rnd(rows, d) * 2 + offset, ht), place(rnd(rows, d) + offset, t)
    gain = lambda: (1 + 0.2 * rnd(d)).to(t).cuda()
    bias = lambda: (0.1 * rnd(d)).to(t).cuda() if biases else None
    a = dict(post_gain=gain() if post else None, post_bias=bias() if post else None, gate=(rnd(gates, d) * 0.7).to(t).cuda() if gates else None,
             pre_gain=gain() if pre else None, pre_bias=bias() if pre else None)
    h_out, z = B.sjd_block_norm(h, y=y, gate_tanh=tanh, scale=scale, kind=kind, eps=eps, **a)
    x, off = y.double(), torch.zeros(rows, d, dtype=torch.float64, device="cuda")
    if post:
        x, off = _norm(x, off, a["post_gain"], a["post_bias"], layer, eps)
    if gates:
        w = a["gate"].double().repeat_interleave(rows // gates, 0)
        w = torch.tanh(w) if tanh else w
        x, off = x * w, off * w.abs() + 4 * E * (x * w).abs()   # (a hyperbolic tangent of the device: two steps)
    want = h.double() + scale * x
    off = scale * off + E * (scale * x).abs() + E * want.abs()
    step = lambda v, dt: v.abs() * (2.0 ** -8 if dt is torch.bfloat16 else E) + 1e-37
    assert ((h_out.double() - want).abs() <= off * 1.01 + step(want, ht)).all()
    if pre:
        want, off = _norm(want, off, a["pre_gain"], a["pre_bias"], layer, eps)
        assert ((z.double() - want).abs() <= off * 1.01 + step(want, t)).all()
    else:
        assert z is None
    return h_out, z


@pytest.mark.gpu
@pytest.mark.parametrize("d", [1, 7, 8, 31, 64, 255, 256, 257, 264, 512, 683, 1000, 1024, 1032, 4096, 4100, 8192, 8193, 11008, 16384, 16392, 32760, 32767, 32768])
@pytest.mark.parametrize("rows", [1, 5])
def test_widths(rows, d):
    for i, (dtype, h_dtype) in enumerate(itertools.product(DT, DT)):
        _check(rows, d, dtype, h_dtype, B.SJD_NORM_RMS if i % 2 else B.SJD_NORM_LAYER, True, rows if i < 2 else 1, i < 1, True, i > 1, seed=i)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [B.SJD_NORM_RMS, B.SJD_NORM_LAYER])
@pytest.mark.parametrize("post,gates,tanh,pre,biases", list(itertools.product([True, False], [0, 1, 4], [True, False], [True, False], [True, False])))
def test_parts_that_are_left_out(kind, post, gates, tanh, pre, biases):
    _check(12, 520, "bf16", "f32", kind, post, gates, tanh, pre, biases, scale=0.7)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", [(513, 4096), (600, 8192), (1000, 16384), (3000, 128), (700, 683)])
def test_many_rows(rows, d):
    _check(rows, d, "bf16", "bf16", B.SJD_NORM_RMS, True, 0, False, True, False)
    _check(rows, d, "f32", "f32", B.SJD_NORM_LAYER, True, rows, True, True, True)


@pytest.mark.gpu
@pytest.mark.parametrize("pad", [1, 8, 24])
def test_strides(pad):
    _check(9, 768, "bf16", "f32", B.SJD_NORM_LAYER, True, 3, False, True, True, pad=pad)


@pytest.mark.gpu
def test_a_mean_far_from_zero_and_entries_without_spread():
    _check(6, 4096, "f32", "f32", B.SJD_NORM_LAYER, True, 0, False, True, False, offset=100.0)
    h = torch.full((3, 96), 5.0, device="cuda")
    assert (B.sjd_block_norm(h, pre_gain=torch.ones(96, device="cuda"), kind=B.SJD_NORM_LAYER)[1] == 0).all()
    assert (B.sjd_block_norm(torch.zeros_like(h), pre_gain=torch.ones(96, device="cuda"))[1] == 0).all()


@pytest.mark.gpu
def test_alone_in_place_and_no_rows():
    g = torch.Generator().manual_seed(4)
    h, y, w = (torch.randn(*s, generator=g).bfloat16().cuda() for s in ((40, 1024), (40, 1024), (1024,)))
    a, b = B.sjd_block_norm(h, y=y, post_gain=w, pre_gain=w)
    h2, y2 = h.clone(), y.clone()
    B.sjd_block_norm(h2, y=y2, post_gain=w, pre_gain=w, h_out=h2, z=y2)
    assert torch.equal(h2, a) and torch.equal(y2, b)
    none, z = B.sjd_block_norm(h.float(), pre_gain=w)   # residual stream in fp32, norm in bf16
    want, off = _norm(h.double(), torch.zeros_like(h.double()), w, None, False, 1e-5)
    assert none is None and z.dtype is torch.bfloat16 and ((z.double() - want).abs() <= off + want.abs() * 2.0 ** -8).all()
    assert B.sjd_block_norm(h[:0], pre_gain=w)[1].shape == (0, 1024)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", [(6001, 512), (700, 4096), (333, 8192)])
def test_many_rows_in_place(rows, d):
    """Enough of them for the kernel that fetches rows ahead: those are read before, or after, nobody writes them."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    h, y, w = (torch.randn(*s, generator=g, device="cuda").bfloat16() for s in ((rows, d), (rows, d), (d,)))
    a, b = B.sjd_block_norm(h, y=y, post_gain=w, pre_gain=w, kind=B.SJD_NORM_LAYER)
    B.sjd_block_norm(h, y=y, post_gain=w, pre_gain=w, kind=B.SJD_NORM_LAYER, h_out=h, z=y)
    assert torch.equal(h, a) and torch.equal(y, b)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", [(5, 200), (5, 203), (7, 1000), (9, 683), (9, 2048), (600, 8192), (9, 10007), (9, 16384), (9, 32768), (6001, 512), (700, 4096)])
@pytest.mark.parametrize("dtype", list(DT))
def test_a_block_whose_output_is_the_residual_stream_itself(rows, d, dtype):
    """y is h, and both outputs go where it was, one of them each time: rows of warps and of blocks, in vectors and one by one, and rows fetched ahead."""
    g = torch.Generator(device="cuda").manual_seed(d)
    h, w = torch.randn(rows, d, generator=g, device="cuda").to(DT[dtype]), torch.randn(d, generator=g, device="cuda").to(DT[dtype])
    kw = dict(post_gain=w, pre_gain=w, kind=B.SJD_NORM_LAYER, scale=0.5)
    a, b = B.sjd_block_norm(h, y=h.clone(), **kw)
    x, y = h.clone(), h.clone()
    _, z = B.sjd_block_norm(x, y=x, h_out=x, **kw)
    assert torch.equal(x, a) and torch.equal(z, b)
    out, _ = B.sjd_block_norm(y, y=y, z=y, **kw)
    assert torch.equal(out, a) and torch.equal(y, b)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", [(9, 264), (9, 2048), (3000, 1024)])
def test_outputs_that_start_on_16_bytes(rows, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    h, y, w = (torch.randn(*s, generator=g, device="cuda") for s in ((rows, d), (rows, d), (d,)))
    a, b = B.sjd_block_norm(h, y=y, post_gain=w, pre_gain=w)
    out, z = (torch.full((rows * d + 8,), 7.0, device="cuda") for _ in range(2))
    B.sjd_block_norm(h, y=y, post_gain=w, pre_gain=w, h_out=out[4:4 + rows * d].view(rows, d), z=z[4:4 + rows * d].view(rows, d))
    for got, want in ((out, a), (z, b)):
        assert torch.equal(got[4:-4].view(rows, d), want) and (got[:4] == 7).all() and (got[-4:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", [(300000, 8192), (70000, 32768)])
def test_rows_behind_four_gigabytes(rows, d):
    """More than 2^31 numbers: the last rows are those of the first, repeated."""
    g = torch.Generator(device="cuda").manual_seed(47)
    part, w = torch.randn(1000, d, generator=g, device="cuda").bfloat16(), torch.randn(d, generator=g, device="cuda").bfloat16()
    h = part.repeat(rows // 1000, 1)
    _, z = B.sjd_block_norm(h, y=h, post_gain=w, pre_gain=w, h_out=h)
    want, off = _norm(part[-50:].double(), torch.zeros(50, d, dtype=torch.float64, device="cuda"), w, None, False, 1e-5)
    want, off = part[-50:].double() + want, off + E * (part[-50:].double().abs() + 2 * want.abs())
    assert ((h[-50:].double() - want).abs() <= 1.01 * off + 2.0 ** -8 * want.abs() + 1e-37).all()
    assert torch.equal(z[:1000], z[-1000:]) and torch.equal(h[:1000], h[-1000:])


@pytest.mark.gpu
def test_rows_do_not_touch_one_another():
    """A NaN or an infinity stays in its row; entries beside the rows stay as they are."""
    h = torch.randn(20, 648, device="cuda").bfloat16()
    y = torch.randn(20, 648, device="cuda").bfloat16()
    w = torch.ones(640, device="cuda", dtype=torch.bfloat16)
    want = B.sjd_block_norm(h[:, :640], y=y[:, :640], post_gain=w, pre_gain=w)
    y[3, 5], h[7, 9] = float("nan"), float("inf")
    out, z = torch.full_like(h, 3.0), torch.full_like(h, 3.0)
    B.sjd_block_norm(h[:, :640], y=y[:, :640], post_gain=w, pre_gain=w, h_out=out[:, :640], z=z[:, :640])
    keep = [i for i in range(20) if i not in (3, 7)]
    assert torch.equal(out[keep, :640], want[0][keep]) and torch.equal(z[keep, :640], want[1][keep])
    assert (out[:, 640:] == 3).all() and (z[:, 640:] == 3).all()
    assert z[3, :640].isnan().all() and out[7, 9].isinf() and z[7, :640].isnan().any()


@pytest.mark.gpu
def test_on_another_stream_and_in_a_graph():
    h, y, w = torch.randn(33, 2048, device="cuda"), torch.randn(33, 2048, device="cuda"), torch.randn(2048, device="cuda")
    want = B.sjd_block_norm(h, y=y, post_gain=w, pre_gain=w)
    out, z = torch.zeros_like(h), torch.zeros_like(h)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sjd_block_norm(h, y=y, post_gain=w, pre_gain=w, h_out=out, z=z)
        B.sjd_block_norm(out, y=z, post_gain=w, pre_gain=w, h_out=out, z=z)
    h.mul_(1.0)
    graph.replay()
    second = B.sjd_block_norm(want[0], y=want[1], post_gain=w, pre_gain=w)
    torch.cuda.synchronize()
    assert torch.equal(out, second[0]) and torch.equal(z, second[1])


@pytest.mark.gpu
def test_binding_refuses_what_does_not_fit():
    h, w = torch.zeros(6, 64, device="cuda"), torch.ones(64, device="cuda")
    for kw in (dict(), dict(pre_gain=w.cpu()), dict(pre_gain=w[:63]), dict(y=h[:5], pre_gain=w), dict(y=h.t(), pre_gain=w),
               dict(y=h, gate=torch.ones(4, 64, device="cuda")), dict(y=h, gate=w), dict(y=h, post_gain=w.bfloat16()), dict(pre_gain=w, h_out=h),
               dict(y=h, z=h), dict(pre_gain=w, z=h.bfloat16()), dict(y=h, h_out=h.bfloat16())):
        with pytest.raises(ValueError):
            B.sjd_block_norm(h, **kw)
    with pytest.raises(B.SJDError):
        B.sjd_block_norm(h, y=h, gate=torch.ones(2, 64, device="cuda"), post_bias=w)
    with pytest.raises(B.SJDError):
        B.sjd_block_norm(h.half(), pre_gain=w)
