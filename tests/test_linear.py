"""sjd_linear: refusals without a GPU, values on one against the formula in 64 bits."""
import itertools
import math

import pytest
import torch

from paper_2410_01699_b200 import binding as B

FAKE = 1 << 20   # an address that no refused call may use
ACTS = {"none": B.SJD_ACT_NONE, "relu": B.SJD_ACT_RELU, "silu": B.SJD_ACT_SILU, "gelu": B.SJD_ACT_GELU, "gelu_tanh": B.SJD_ACT_GELU_TANH}


def _call(**kw):
    a = dict(rows=4, n=64, k=64, x=FAKE, xs=64, w=FAKE, up=None, ws=64, bias=None, bias_up=None, act=0, residual=None, rs=64, out=FAKE, os=64,
             status=None)
    a.update(kw)
    return B.lib().sjd_linear(*a.values(), None)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), B.SJD_ERR_BAD_ARG), (dict(n=0), B.SJD_ERR_BAD_ARG), (dict(k=0), B.SJD_ERR_BAD_ARG), (dict(x=None), B.SJD_ERR_BAD_ARG),
    (dict(w=None), B.SJD_ERR_BAD_ARG), (dict(out=None), B.SJD_ERR_BAD_ARG), (dict(bias_up=FAKE), B.SJD_ERR_BAD_ARG), (dict(xs=56), B.SJD_ERR_BAD_ARG),
    (dict(ws=56), B.SJD_ERR_BAD_ARG), (dict(os=63), B.SJD_ERR_BAD_ARG), (dict(residual=FAKE, rs=63), B.SJD_ERR_BAD_ARG), (dict(xs=68), B.SJD_ERR_BAD_ARG),
    (dict(ws=65), B.SJD_ERR_BAD_ARG), (dict(x=FAKE + 8), B.SJD_ERR_BAD_ARG), (dict(w=FAKE + 2), B.SJD_ERR_BAD_ARG), (dict(up=FAKE + 8), B.SJD_ERR_BAD_ARG),
    (dict(out=FAKE + 1), B.SJD_ERR_BAD_ARG), (dict(bias=FAKE + 1), B.SJD_ERR_BAD_ARG), (dict(status=FAKE + 2), B.SJD_ERR_BAD_ARG),
    (dict(act=5), B.SJD_ERR_UNSUPPORTED), (dict(act=-1), B.SJD_ERR_UNSUPPORTED), (dict(n=(1 << 21) + 1, os=1 << 22), B.SJD_ERR_CAPACITY),
    (dict(k=(1 << 28) + 8, xs=1 << 29, ws=1 << 29), B.SJD_ERR_CAPACITY), (dict(rows=0, x=None, out=None), B.SJD_OK)])
def test_refusals(change, status):
    assert _call(**change) == status


def test_binding_refuses_tensors_of_the_host():
    with pytest.raises(ValueError):
        B.sjd_linear(torch.zeros(2, 8), torch.zeros(3, 8))


def _act(v, name):
    if name == "relu":
        return v.clamp(min=0)
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return v * torch.special.ndtr(v)
    if name == "gelu_tanh":
        return v * torch.sigmoid((8 / math.pi) ** 0.5 * (v + 0.044715 * v ** 3))
    return v


def _off(sums, k, v, name):
    """How far act(v) may be off in fp32.  Products of bf16 numbers are exact; tensor memory takes 16 of them a step and rounds towards zero
    (2^-23 of the magnitudes so far), up to eight ranges and a bias are added.  A derivative of an activation is at most 1.13; its own evaluation (an
    exponential of up to 2^-21 of itself for each unit of its argument, which is at most 88, a quotient or a tangent) leaves 2^-18 of it, or
    of v where it cancels."""
    off = 1.13 * (k / 16 + 12) * 2.0 ** -23 * sums
    return off if name in ("none", "relu") else off + 2.0 ** -18 * v.abs()


def _check(rows, n, k, act="none", gated=False, bias=False, residual=False, seed=0, pad=0, in_place=False, out_pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    wide = -(-k // 8) * 8 + 8 * pad
    x, w = rnd(rows, wide).bfloat16()[:, :k], (rnd(n, wide) * k ** -0.5).bfloat16()[:, :k]
    up = (rnd(n, wide) * k ** -0.5).bfloat16()[:, :k] if gated else None
    b, c = (rnd(n) * 0.5).bfloat16() if bias else None, (rnd(n) * 0.5).bfloat16() if bias and gated else None
    whole = rnd(rows, n + out_pad).bfloat16()
    r = whole[:, :n] if in_place else rnd(rows, n).bfloat16() if residual else None
    kept, before = r.clone() if r is not None else None, whole.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = B.sjd_linear(x, w, w_up=up, bias=b, bias_up=c, act=ACTS[act], residual=r, out=whole[:, :n], status=status)
    pre = x.double() @ w.double().t()
    sums = x.double().abs() @ w.double().abs().t()
    if b is not None:
        pre, sums = pre + b.double(), sums + b.double().abs()
    want, off = _act(pre, act), _off(sums, k, pre, act)
    if gated:
        u = x.double() @ up.double().t()
        s = x.double().abs() @ up.double().abs().t()
        if c is not None:
            u, s = u + c.double(), s + c.double().abs()
        off = off * (u.abs() + _off(s, k, u, "none")) + want.abs() * _off(s, k, u, "none")
        want = want * u
    if kept is not None:
        want = want + kept.double()
    off = off + 3 * 2.0 ** -24 * want.abs()
    err = (out.double() - want).abs()
    bad = err > 1.001 * off + want.abs() * 2.0 ** -8 + 1e-37
    assert status.item() == 0 and not bad.any(), "%d of %d, first at %s" % (bad.sum(), bad.numel(), bad.nonzero()[0].tolist())
    if out_pad:
        assert torch.equal(whole[:, n:], before[:, n:])


SMALL = [(1, 1, 1), (1, 512, 512), (2, 8, 16), (3, 130, 70), (15, 683, 256), (16, 128, 64), (17, 129, 65), (31, 1408, 512), (33, 64, 2000),
         (48, 1000, 683), (63, 127, 63), (64, 4096, 4096), (5, 20000, 128), (1, 40000, 64), (64, 65536, 72)]
PAIRS = [(65, 1, 8), (65, 256, 64), (80, 300, 130), (100, 4096, 512), (127, 511, 1000), (128, 128, 8192), (129, 257, 96), (200, 640, 4096),
         (255, 1024, 64), (256, 4096, 11008), (257, 512, 512), (300, 129, 63), (511, 2000, 1408), (1063, 1536, 512), (1500, 4100, 100), (4223, 260, 264)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,k", SMALL + PAIRS)
@pytest.mark.parametrize("gated", [False, True])
def test_sizes(rows, n, k, gated):
    _check(rows, n, k, "silu" if gated else "none", gated)
    _check(rows, n, k, "gelu", gated, bias=True, residual=True, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,k", [(7, 200, 136), (64, 96, 1000), (90, 200, 136), (300, 600, 328), (2000, 5000, 64)])
@pytest.mark.parametrize("act,gated,bias,residual", list(itertools.product(ACTS, [False, True], [False, True], [False, True])))
def test_epilogues(rows, n, k, act, gated, bias, residual):
    _check(rows, n, k, act, gated, bias, residual)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 200])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
def test_tails_of_activations(rows, act, gated):
    """Sums that are exact (one product, by 1), where 1 + erf and 1 + tanh have cancelled: the error is the activation's own, relative to it.  Arguments of
    the exponentials are up to 2 u = 87 with up to 8 roundings, 87 * 8 * 2^-24, and exponentials off by 2 + 1.2 * 87 units of 2^-23; in GELU the argument is v^2 / 2 = 50
    and the rest of the complementary error function off by 2^-17; quotients and products 2^-18.  So 2^-14, and the output's rounding."""
    v = torch.cat((torch.linspace(-10, -3, 701), torch.linspace(-3, 10, 400))).bfloat16().cuda()
    x, w = torch.zeros(rows, 8, device="cuda").bfloat16(), torch.zeros(v.numel(), 8, device="cuda").bfloat16()
    x[:, 3], w[:, 3] = 1, v
    out = B.sjd_linear(x, w, w_up=torch.where(w == 0, w, torch.full_like(w, 1024.0)) if gated else None, act=ACTS[act])
    e = v.double()
    want = e * torch.special.erfc(-e * 0.5 ** 0.5) / 2 if act == "gelu" else _act(e, act)
    want = want * torch.where(v == 0, 0.0, 1024.0) if gated else want
    err = (out.double() - want).abs()
    assert (err <= (2.0 ** -8 + 2.0 ** -14) * want.abs()).all(), "%.3g of it" % (err / want.abs().clamp(min=1e-300)).max()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,k", [(1, 40, 24), (9, 100, 120), (70, 100, 120), (600, 300, 64)])
def test_strides_and_in_place(rows, n, k):
    _check(rows, n, k, pad=3, out_pad=5, residual=True)
    _check(rows, n, k, "silu", True, pad=1, in_place=True, out_pad=1)
    _check(rows, n, k, in_place=True, bias=True)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", range(1, 65))
def test_every_number_of_few_rows(rows):
    _check(rows, 264, 200, "silu", rows % 2 == 0, residual=True, seed=rows)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", list(range(66, 300, 13)) + [511, 512, 513, 1023, 1024, 1025])
def test_more_rows(rows):
    _check(rows, 700, 456, "gelu_tanh", rows % 2 == 0, bias=True, seed=rows)


@pytest.mark.gpu
def test_what_lies_behind_the_entries_does_not_matter():
    """NaN behind k in a row, and rows and features behind the last."""
    for rows, n, k in ((5, 30, 20), (70, 300, 100), (900, 900, 36)):
        g = torch.Generator(device="cuda").manual_seed(3)
        x, w = (torch.randn(m, k + 20 & ~7, generator=g, device="cuda").bfloat16() for m in (rows + 9, n + 9))
        want = B.sjd_linear(x[:rows, :k].clone()[:, :k] if k % 8 == 0 else x[:rows, :k], w[:n, :k])
        x[:, k:], w[:, k:], x[rows:], w[n:] = (float("nan"),) * 4
        out = torch.full((rows + 3, n), 2.0, device="cuda").bfloat16()
        B.sjd_linear(x[:rows, :k], w[:n, :k], out=out[:rows])
        assert torch.equal(out[:rows], want) and (out[rows:] == 2).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [6, 100, 1100])
def test_nan_and_infinity_stay_in_their_row(rows):
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w = (torch.randn(m, 128, generator=g, device="cuda").bfloat16() for m in (rows, 200))
    want = B.sjd_linear(x, w)
    x[2, 7], x[4, 9] = float("nan"), float("inf")
    out = B.sjd_linear(x, w)
    keep = [i for i in range(rows) if i not in (2, 4)]
    assert torch.equal(out[keep], want[keep]) and out[2].isnan().all() and not out[4].isfinite().any()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,k,gated", [(8, 512, 4096, False), (8, 512, 4096, True), (200, 512, 4096, True), (700, 3000, 512, False)])
def test_the_same_bits_every_time_in_a_graph_and_on_another_stream(rows, n, k, gated):
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w, u = (torch.randn(m, k, generator=g, device="cuda").bfloat16() for m in (rows, n, n))
    call = lambda out=None: B.sjd_linear(x, w, w_up=u if gated else None, act=B.SJD_ACT_SILU, out=out)
    want = call()
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for _ in range(20):
            out.zero_()
            call(out)
            assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call()
        z = B.sjd_linear(y, y[:16].clone())   # (right behind, on what the first wrote)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(z, B.sjd_linear(want, want[:16].clone()))


@pytest.mark.gpu
def test_outputs_behind_four_gigabytes():
    """More than 2^31 numbers: rows from both ends beside a call of their own."""
    g = torch.Generator(device="cuda").manual_seed(46)
    x, w = torch.randn(66000, 64, generator=g, device="cuda").bfloat16(), (torch.randn(32768, 64, generator=g, device="cuda") / 8).bfloat16()
    out = B.sjd_linear(x, w)
    for rows in (slice(0, 100), slice(65500, 65600), slice(65950, 66000)):
        v = x[rows].double() @ w.double().t()
        off = _off(x[rows].double().abs() @ w.double().abs().t(), 64, v, "none")
        assert ((out[rows].double() - v).abs() <= 1.001 * off + 2.0 ** -8 * v.abs() + 1e-37).all()


@pytest.mark.gpu
def test_no_rows():
    assert B.sjd_linear(torch.zeros(0, 64, device="cuda").bfloat16(), torch.zeros(8, 64, device="cuda").bfloat16()).shape == (0, 8)


@pytest.mark.gpu
def test_binding_refuses_what_does_not_fit():
    x, w = torch.zeros(6, 64, device="cuda").bfloat16(), torch.zeros(32, 64, device="cuda").bfloat16()
    for kw in (dict(w=w[:, :56]), dict(w=w.float()), dict(w=w.cpu()), dict(w_up=w[:31]), dict(bias=x[0]), dict(residual=x), dict(out=x),
               dict(bias=torch.zeros(32, device="cuda")), dict(x=x.t()), dict(w_up=torch.zeros(32, 128, device="cuda").bfloat16()[:, :64])):
        with pytest.raises(ValueError):
            B.sjd_linear(**{**dict(x=x, w=w), **kw})
    for kw in (dict(x=x.float()), dict(x=x[:, 4:], w=w[:, 4:]), dict(bias_up=w[:, 0].contiguous()), dict(act=7)):
        with pytest.raises(B.SJDError):
            B.sjd_linear(**{**dict(x=x, w=w), **kw})
