"""sjd_block_norm, sjd_linear and sjd_pool_attention_shared together: decoding steps of a small decoder whose sequences share a prompt, eagerly
and as a captured graph.  Every stage against its formula in 64 bits of what it was given."""
import numpy as np
import pytest
import torch

from paper_2410_01699_b200 import binding as B
from tests import test_block_norm as N, test_linear as L, test_pool_shared as S

D, HEADS, KVH, HD, FF, VOCAB, LAYERS, PROMPT = 512, 8, 2, 64, 1408, 1000, 2, 300


def _weights():
    g = torch.Generator(device="cuda").manual_seed(40)
    w = lambda n, k: (torch.randn(n, k, generator=g, device="cuda") * k ** -0.5).bfloat16()
    gain = lambda: (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).bfloat16()
    layers = [dict(g1=gain(), qkv=w((HEADS + 2 * KVH) * HD, D), o=w(D, HEADS * HD), g2=gain(), gate=w(FF, D), up=w(FF, D), down=w(D, FF)) for _ in range(LAYERS)]
    return layers, gain(), w(VOCAB, D)


def _step(weights, pool, h, pos, window, begin, status, kept=None):
    """One pass over the layers; kept: a list that gets every stage with what it was given."""
    layers, last, head = weights
    keep = (lambda *a: kept.append(a)) if kept is not None else lambda *a: None

    def norm(h, y, gain):
        out, z = B.sjd_block_norm(h, y=y, pre_gain=gain)
        keep("norm", h, y, gain, out, z)
        return (h if out is None else out), z

    def linear(x, w, **kw):
        out = B.sjd_linear(x, w, status=status, **kw)
        keep("linear", x, w, kw, out)
        return out
    y = None
    for i, w in enumerate(layers):
        h, z = norm(h, y, w["g1"])
        heads = linear(z, w["qkv"]).unflatten(1, (-1, HD))
        q = B.sjd_pool_append(pool, i, heads[:, HEADS:HEADS + KVH], heads[:, HEADS + KVH:], pos, window, q=heads[:, :HEADS], rope=B.make_rope_cfg((HD // 2,)))
        o = B.sjd_pool_attention_shared(pool, i, q, pos, window, group_begin=begin)
        keep("attention", i, q, o)
        h, z = norm(h, linear(o.flatten(1), w["o"]), w["g2"])
        y = linear(linear(z, w["gate"], w_up=w["up"], act=B.SJD_ACT_SILU), w["down"])
    return linear(norm(h, y, last)[1], head)


def _hold(kept, pool, pos, window, short):
    for name, *a in kept:
        if name == "norm":
            h, y, gain, out, z = a
            x, off = h.double(), torch.zeros_like(h, dtype=torch.float64)
            if y is not None:
                x = x + y.double()
                off = N.E * x.abs()
                assert ((out.double() - x).abs() <= 1.01 * off + 1e-37).all()
            want, off = N._norm(x, off, gain, None, False, 1e-5)
            assert ((z.double() - want).abs() <= 1.01 * off + 2.0 ** -8 * want.abs() + 1e-37).all()
        elif name == "linear":
            x, w, kw, out = a
            k = w.shape[1]
            both = lambda w: (x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t())
            v, sums = both(w)
            act = "silu" if kw else "none"
            want, off = L._act(v, act), L._off(sums, k, v, act)
            if kw:
                u, s = both(kw["w_up"])
                off = off * (u.abs() + L._off(s, k, u, "none")) + want.abs() * L._off(s, k, u, "none")
                want = want * u
            assert ((out.double() - want).abs() <= 1.001 * off + (2.0 ** -8 + 3 * 2.0 ** -24) * want.abs() + 1e-37).all()
        else:
            i, q, o = a
            if short:
                assert torch.equal(o, B.sjd_pool_attention(pool, i, q, pos, window))
            else:
                S._within(pool, o, q, pos.tolist(), window, layer=i)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,window,pages", [(5, 4, S.LONG), (24, 1, S.LONG), (3, 40, S.LONG), (2, 1, 8)])
def test_steps_of_a_decoder(batch, window, pages):
    weights, status = _weights(), torch.zeros(1, dtype=torch.int32, device="cuda")
    pool = B.CachePool.empty(5 + 4 * batch, batch, pages, LAYERS, KVH, HD)
    g = torch.Generator(device="cuda").manual_seed(41)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    # a prompt, and sequences that share its pages (but the last, which they get copies of when they write)
    B.sjd_pool_reserve(pool, S._i32([0]), S._i32([0]), S._i32([PROMPT]))
    for i in range(LAYERS):
        B.sjd_pool_append(pool, i, rnd(PROMPT, KVH, HD).bfloat16(), rnd(PROMPT, KVH, HD).bfloat16(), S._i32(list(range(PROMPT))), PROMPT)
    children = list(range(1, batch))
    B.sjd_pool_fork(pool, S._i32([0] * len(children)), S._i32(children), S._i32([PROMPT] * len(children)))
    begin = S._i32([0, batch])
    steps = 3
    at = [PROMPT + np.arange(window) + s * window for s in range(steps)]
    B.sjd_pool_reserve(pool, S._i32(list(range(batch))), S._i32([PROMPT] * batch), S._i32([PROMPT + steps * window] * batch))
    h, pos = rnd(batch * window, D), S._i32([0] * (batch * window))
    # a step that is captured, replayed on its own inputs and beside one that is not
    pos.copy_(S._i32(np.tile(at[0], batch).tolist()))
    _step(weights, pool, h, pos, window, begin, status)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _step(weights, pool, h, pos, window, begin, status)
    for s in range(steps):
        h.copy_(rnd(batch * window, D))
        pos.copy_(S._i32(np.tile(at[s], batch).tolist()))
        kept = []
        logits = _step(weights, pool, h, pos, window, begin, status, kept)
        _hold(kept, pool, pos, window, pages != S.LONG)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, logits)
    assert status.item() == 0 and pool.fault() == 0
    shared = pool.table[:, :PROMPT // 64]
    assert (shared == shared[:1]).all() and (pool.table[:, PROMPT // 64].unique().numel() == batch)


@pytest.mark.gpu
def test_calls_on_two_streams_at_once():
    """Calls of every kernel beside one another, attention with a workspace for each stream: the bits of calls one after the other."""
    g = torch.Generator(device="cuda").manual_seed(42)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    pool, lens = S._filled([(6, [600, 500, 430]), (3, [300, 210])], 1, 2, 128, 43)
    q, at, begin = rnd(len(lens) * 20, 8, 128), S._i32(S._window_pos(lens, 20)), S._i32([0, 3, 5])
    short = B.CachePool(pool.pages, pool.exps, pool.table[:, :10].contiguous(), pool.refs)
    x, w, up, gain = rnd(700, 1024), rnd(1024, 1024) / 32, rnd(1024, 1024) / 32, rnd(1024)
    nbytes = int(B.lib().sjd_pool_attention_shared_workspace_bytes(pool.ref, len(lens), 20, 8))

    def work(ws):
        return [B.sjd_pool_attention_shared(pool, 0, q, at, 20, group_begin=begin, ws=ws), B.sjd_linear(x, w, w_up=up, act=B.SJD_ACT_SILU),
                B.sjd_block_norm(x, y=x, pre_gain=gain)[1], B.sjd_linear(x[:33], w, residual=x[:33]), B.sjd_pool_attention_shared(short, 0, q, at, 20, group_begin=begin, ws=ws),
                B.sjd_linear(x[:200], w), B.sjd_block_norm(x.repeat(6, 1), pre_gain=gain)[1]]
    spaces = [torch.empty(nbytes, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = work(spaces[0])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in spaces], []
    for _ in range(5):
        for stream, ws in zip(streams, spaces):
            with torch.cuda.stream(stream):
                got.append(work(ws))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for each in got for a, b in zip(each, want)) and pool.fault() == 0 and short.fault() == 0
