"""The operators of a server's own decoder loop beside the 8-bit paged cache: what a call of each computes, in plain torch, and the
cases that are timed.

  linear     sjd_linear: out = residual + act(x W^T + b) [* (x U^T + c)], bf16, from one row to whole prompts
  norm       sjd_block_norm: h' = h + scale * gate * norm(y), z = norm(h'): the norm after a block, its gate, the residual and the
             norm before the next block
  attention  sjd_pool_attention_shared: window queries over the pool, causal; the pages that the sequences of a group share (a
             common prompt, an image's streams) are attended once for all of the group's rows

Shapes follow the repository's own models: widths of 4096 with SwiGLU of 11008 and 14336 and of 512 with 1408, 32 heads of 128
with 32 or 8 kv heads and 8 heads of 64 with 2, windows of up to 64, prompts of up to 4224 positions, and longer ones.
"""
import math

import torch

own = False

PAGE, BLOCK = 64, 16
# heads, kv heads, head_dim, width, hidden width of the feed-forward
MODELS = {"7b": (32, 32, 128, 4096, 11008), "8b-gqa": (32, 8, 128, 4096, 14336), "small": (8, 2, 64, 512, 1408)}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def listed():
    lin = dict(kind="linear", act="none", gated=False, bias=False, residual=False)
    norm = dict(kind="norm", norm="rms", post=True, gate="none", tanh=False, pre=True, scale=1.0)
    att = dict(kind="attention")
    return [
        # the smallest call: the output projection of one token of the small model, added to the residual
        dict(lin, name="lin_one_token", rows=1, k=512, n=512, residual=True),
        # gate and up projection of a serving batch, a token each
        dict(lin, name="lin_swiglu_b32", rows=32, k=4096, n=14336, act="silu", gated=True),
        # down projection of eight windows of 32 drafts, added to the residual
        dict(lin, name="lin_down_8x32", rows=256, k=11008, n=4096, residual=True),
        # queries, keys and values of a prompt that holds an image, with a bias
        dict(lin, name="lin_qkv_prompt", rows=1063, k=4096, n=6144, bias=True),
        # gate and up projection of a whole image: the largest product
        dict(lin, name="lin_swiglu_image", rows=4223, k=4096, n=14336, act="silu", gated=True),
        # one token of the small model: norms on both sides of the residual
        dict(norm, name="norm_one_token", rows=1, d=512, dtype="bf16", h_dtype="bf16"),
        # windows of eight sequences, a gate for each sequence, residual stream in fp32
        dict(norm, name="norm_8x32_gate", rows=256, d=4096, dtype="bf16", h_dtype="f32", gate="sequence", tanh=True, seqs=8),
        # the prompts of four images
        dict(norm, name="norm_prompt", rows=4 * 4223, d=4096, dtype="bf16", h_dtype="bf16", norm="layer", gate="channel", scale=0.5),
        # two sequences of a short prompt, a token each: launches and latency
        dict(att, name="att_small", model="small", groups=1, members=2, window=1, shared=128, length=217),
        # sixteen images of one prompt, windows of 32 drafts
        dict(att, name="att_images_16x32", model="8b-gqa", groups=1, members=16, window=32, shared=1024, length=2311),
        # two prompts that hold an image each, eight answers to both, every head its own keys
        dict(att, name="att_prompts_2x8", model="7b", groups=2, members=8, window=16, shared=4224, length=4601),
        # many answers to one long document, a token each
        dict(att, name="att_document_64", model="8b-gqa", groups=1, members=64, window=1, shared=32768, length=33003),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "norm", "attention", "attention"))
    model = rng.choice(tuple(MODELS))
    heads, kv_heads, hd, width, hidden = MODELS[model]
    if kind == "linear":
        k, n = rng.choice(((width, hidden), (hidden, width), (width, (heads + 2 * kv_heads) * hd), (_log_int(rng, 16, 12000), _log_int(rng, 8, 15000))))
        gated = rng.random() < 0.4
        rows = _log_int(rng, 1, 4223)
        rows = max(1, min(rows, 4223 * 4096 * 28672 // (k * n * (2 if gated else 1))))
        return dict(kind=kind, rows=rows, k=k, n=n, act=rng.choice(ACTS[1:] if gated else ACTS), gated=gated, bias=rng.random() < 0.4,
                    residual=rng.random() < 0.4)
    if kind == "norm":
        d = rng.choice((width, _log_int(rng, 8, 16384)))
        rows = max(1, min(_log_int(rng, 1, 16892), 16892 * 4096 // d))
        gate = rng.choice(("none", "channel", "sequence"))
        post = rng.random() < 0.7
        seqs = rng.choice([s for s in (1, 2, 3, 4, 8, 16) if rows % s == 0])
        return dict(kind=kind, rows=rows, d=d, dtype=rng.choice(("bf16", "bf16", "f32")), h_dtype=rng.choice(("bf16", "f32")),
                    norm=rng.choice(("rms", "layer")), post=post, gate=gate, tanh=gate != "none" and rng.random() < 0.5, seqs=seqs,
                    pre=rng.random() < 0.8, scale=rng.choice((1.0, 0.5, 1.4)))
    groups, members = rng.choice((1, 1, 2, 3)), _log_int(rng, 1, 64)
    window = _log_int(rng, 1, 64)
    members = max(1, min(members, 1024 // (window * groups)))
    shared = PAGE * _log_int(rng, 1, 512) if rng.random() < 0.85 else 0
    length = shared + window + _log_int(rng, 1, 2000)
    # no more positions in the pool, and no more scores, than the largest listed cases
    rows = groups * members * window
    shared = min(shared, (1 << 28) // (heads * rows) // PAGE * PAGE)
    length = max(shared + window, min(length, (1 << 28) // (heads * rows), shared + (1 << 18) // (groups * members * kv_heads) * 8))
    return dict(kind=kind, model=model, groups=groups, members=members, window=window, shared=shared, length=length)


# ---------------------------------------------------------------------------------------------------------------- states
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    if case["kind"] == "linear":
        rows, k, n = case["rows"], case["k"], case["n"]
        # (rows of matrices start on 16 bytes: a width that is no multiple of 8 lies in a wider one)
        wide = -(-k // 8) * 8
        s = {"x": randn(rows, wide).bfloat16()[:, :k], "w": (randn(n, wide) * k ** -0.5).bfloat16()[:, :k], "w_up": None, "bias": None,
             "bias_up": None, "residual": None, "out": torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")}
        if case["gated"]:
            s["w_up"] = (randn(n, wide) * k ** -0.5).bfloat16()[:, :k]
        if case["bias"]:
            s["bias"] = (randn(n) * 0.3).bfloat16()
            s["bias_up"] = (randn(n) * 0.3).bfloat16() if case["gated"] else None
        if case["residual"]:
            s["residual"] = randn(rows, n).bfloat16()
    elif case["kind"] == "norm":
        rows, d, t, ht = case["rows"], case["d"], DTYPES[case["dtype"]], DTYPES[case["h_dtype"]]
        layer = case["norm"] == "layer"
        gain = lambda: (1 + 0.2 * randn(d)).to(t)
        s = {"h": (randn(rows, d) * 2).to(ht), "y": (randn(rows, d) * torch.exp(0.5 * randn(rows, 1))).to(t), "post_gain": None, "post_bias": None,
             "gate": None, "pre_gain": None, "pre_bias": None, "h_out": torch.empty(rows, d, dtype=ht, device="cuda"),
             "z": torch.empty(rows, d, dtype=t, device="cuda") if case["pre"] else None}
        if case["post"]:
            s["post_gain"], s["post_bias"] = gain(), (0.1 * randn(d)).to(t) if layer else None
        if case["gate"] != "none":
            s["gate"] = (randn(case["seqs"] if case["gate"] == "sequence" else 1, d) * 0.7).to(t)
        if case["pre"]:
            s["pre_gain"], s["pre_bias"] = gain(), (0.1 * randn(d)).to(t) if layer else None
    else:
        heads, kv_heads, hd = MODELS[case["model"]][:3]
        groups, members, window, shared = case["groups"], case["members"], case["window"], case["shared"] // PAGE
        batch, lens = groups * members, _lens(case)
        per_seq = -(-case["length"] // PAGE)
        counts = [-(-n // PAGE) - shared for n in lens]
        n_pages = groups * shared + sum(counts) + 1
        s = {"pages": torch.empty(n_pages, 1, 2, kv_heads, PAGE, hd, dtype=torch.float8_e4m3fn, device="cuda"),
             "exps": torch.randint(-8, -5, (n_pages, 1, 2, kv_heads, PAGE // BLOCK), generator=gen, device="cuda").to(torch.int8),
             "table": torch.full((batch, per_seq), -1, dtype=torch.int32, device="cuda"),
             "refs": torch.zeros(n_pages, dtype=torch.int32, device="cuda")}
        for i in range(0, n_pages, 256):   # entries as 16 normal rows fill them: a largest one of 200 to 448
            s["pages"][i:i + 256] = randn(*s["pages"][i:i + 256].shape).mul_(70).clamp_(-448, 448).to(torch.float8_e4m3fn)
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        at = 0
        for g in range(groups):
            s["table"][g * members:(g + 1) * members, :shared] = order[at:at + shared]
            s["refs"][order[at:at + shared].long()] = members
            at += shared
        for b, c in enumerate(counts):
            s["table"][b, shared:shared + c] = order[at:at + c]
            s["refs"][order[at:at + c].long()] = 1
            at += c
        if shared:
            s["exps"][s["table"][:, 0].long(), :, 1, :, 0] -= 3   # (values of first tokens are small)
        pos = torch.arange(window, device="cuda")[None] + torch.tensor(lens, device="cuda")[:, None] - window
        s["in_pos"] = pos.to(torch.int32).reshape(-1).contiguous()
        s["group_begin"] = torch.arange(0, batch + 1, members, dtype=torch.int32, device="cuda")
        s["q"] = (randn(batch * window, heads, hd) * 1.3).bfloat16()
        s["out"] = torch.empty_like(s["q"])
        if own:
            from paper_2410_01699_b200 import binding as B
            s["pool"] = B.CachePool(s["pages"], s["exps"], s["table"], s["refs"])
    s["case"] = dict(case)
    return s


def _lens(case):
    """Lengths of the sequences: they share a prefix and have come to different places behind it."""
    batch, least = case["groups"] * case["members"], case["shared"] + case["window"]
    return [max(least, case["length"] - b * (case["length"] - least) // (2 * batch)) for b in range(batch)]


# ------------------------------------------------------------------------------------------------------------------ runs
def run(state):
    return {"linear": _linear, "norm": _norm, "attention": _attention}[state["case"]["kind"]](state)


def _act(x, name):
    if name == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x))
    if name == "silu":
        return x / (1 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh((2 / math.pi) ** 0.5 * (x + 0.044715 * x * x * x)))
    return x


def _linear(s):
    c = s["case"]
    if own:
        from paper_2410_01699_b200 import binding as B
        return B.sjd_linear(s["x"], s["w"], w_up=s["w_up"], bias=s["bias"], bias_up=s["bias_up"],
                            act=getattr(B, "SJD_ACT_" + c["act"].upper()), residual=s["residual"], out=s["out"])
    x = s["x"].float()
    y = torch.matmul(x, s["w"].float().t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _act(y, c["act"])
    if s["w_up"] is not None:
        up = torch.matmul(x, s["w_up"].float().t())
        y = y * (up + s["bias_up"].float() if s["bias_up"] is not None else up)
    if s["residual"] is not None:
        y = s["residual"].float() + y
    return s["out"].copy_(y)


def _norm(s):
    c = s["case"]
    if own:
        from paper_2410_01699_b200 import binding as B
        return B.sjd_block_norm(s["h"], y=s["y"], post_gain=s["post_gain"], post_bias=s["post_bias"], gate=s["gate"], gate_tanh=c["tanh"],
                                scale=c["scale"], pre_gain=s["pre_gain"], pre_bias=s["pre_bias"],
                                kind=B.SJD_NORM_LAYER if c["norm"] == "layer" else B.SJD_NORM_RMS, eps=1e-5, h_out=s["h_out"], z=s["z"])

    def norm(x, gain, bias):
        if c["norm"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gain.float()
        return x if bias is None else x + bias.float()

    t = s["y"].float()
    if s["post_gain"] is not None:
        t = norm(t, s["post_gain"], s["post_bias"])
    if s["gate"] is not None:
        g = s["gate"].float()
        g = torch.tanh(g) if c["tanh"] else g
        t = (t.view(g.shape[0], -1, c["d"]) * g[:, None]).view(-1, c["d"])
    h = s["h"].float() + c["scale"] * t
    s["h_out"].copy_(h)
    if s["pre_gain"] is None:
        return s["h_out"], None
    return s["h_out"], s["z"].copy_(norm(h, s["pre_gain"], s["pre_bias"]))


def _attention(s):
    c = s["case"]
    if own:
        from paper_2410_01699_b200 import binding as B
        return B.sjd_pool_attention_shared(s["pool"], 0, s["q"], s["in_pos"], c["window"], group_begin=s["group_begin"], out=s["out"])
    m, heads, hd = s["q"].shape
    window, groups, members = c["window"], c["groups"], c["members"]
    batch, kv_heads, per_seq, shared = groups * members, s["pages"].shape[3], s["table"].shape[1], c["shared"]

    def keys_and_values(table):   # [K|V][sequence][kv head][position][hd]
        at = table.clamp(min=0).long()
        scale = torch.exp2(s["exps"][at][:, :, 0].float())
        kv = s["pages"][at][:, :, 0].float().view(*at.shape, 2, kv_heads, PAGE // BLOCK, BLOCK, hd) * scale[..., None, None]
        return kv.permute(2, 0, 3, 1, 4, 5, 6).reshape(2, at.shape[0], kv_heads, at.shape[1] * PAGE, hd)

    # scores of the shared positions for all rows of a group, and of the sequences' own
    q = s["q"].float().view(groups, members, window, kv_heads, heads // kv_heads, hd).permute(0, 3, 1, 2, 4, 5)
    first = keys_and_values(s["table"][::members, :shared // PAGE])
    each = window * (heads // kv_heads)   # rows of a sequence and kv head
    a = torch.matmul(q.reshape(groups, kv_heads, members * each, hd), first[0].transpose(-1, -2)) / math.sqrt(hd)
    a = a.view(groups, kv_heads, members, each, shared).transpose(1, 2).reshape(batch, kv_heads, each, shared)
    rest = keys_and_values(s["table"][:, shared // PAGE:])
    b = torch.matmul(q.transpose(1, 2).reshape(batch, kv_heads, each, hd), rest[0].transpose(-1, -2)) / math.sqrt(hd)
    key = torch.arange(rest.shape[3], device="cuda") + shared
    seen = key <= s["in_pos"].view(batch, 1, window, 1, 1)
    b = b.view(batch, kv_heads, window, heads // kv_heads, key.numel()).masked_fill(~seen, -math.inf).view(batch, kv_heads, each, key.numel())
    top = b.amax(-1, keepdim=True) if shared == 0 else torch.maximum(a.amax(-1, keepdim=True), b.amax(-1, keepdim=True))
    a, b = torch.exp(a - top), torch.exp(b - top)
    total = a.sum(-1, keepdim=True) + b.sum(-1, keepdim=True)
    out = torch.matmul(b, rest[1])
    a = a.view(groups, members, kv_heads, each, shared).transpose(1, 2).reshape(groups, kv_heads, members * each, shared)
    out = out + torch.matmul(a, first[1]).view(groups, kv_heads, members, each, hd).transpose(1, 2).reshape(out.shape)
    out = (out / total).view(batch, kv_heads, window, heads // kv_heads, hd).permute(0, 2, 1, 3, 4).reshape(m, heads, hd)
    return s["out"].copy_(out)


# ------------------------------------------------------------------------------------------------------------------ work
def work(case):
    if case["kind"] == "linear":
        rows, k, n, many = case["rows"], case["k"], case["n"], 2 if case["gated"] else 1
        return {"bytes": 2 * (rows * k + many * n * k + rows * n * (2 if case["residual"] else 1) + case["bias"] * many * n),
                "flops": 2.0 * rows * k * n * many}
    if case["kind"] == "norm":
        rows, d, t, ht = case["rows"], case["d"], DTYPES[case["dtype"]].itemsize, DTYPES[case["h_dtype"]].itemsize
        return {"bytes": rows * d * (t + 2 * ht + (t if case["pre"] else 0)), "flops": 12.0 * rows * d}
    heads, kv_heads, hd = MODELS[case["model"]][:3]
    rows = case["groups"] * case["members"] * case["window"]
    keys = case["groups"] * case["shared"] + sum(n - case["shared"] for n in _lens(case))
    pairs = sum(sum(range(n - case["window"] + 1, n + 1)) for n in _lens(case))
    return {"bytes": keys * 2 * kv_heads * hd * (1 + 1 / (BLOCK * hd)) + 4 * rows * heads * hd + rows * 4, "flops": 4.0 * hd * heads * pairs}


# ----------------------------------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The definition in 64 bits, one sequence at a time where there are sequences."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f = lambda t: None if t is None else t.double()
    if case["kind"] == "linear":
        pre = torch.einsum("mk,nk->mn", f(s["x"]), f(s["w"]))
        pre = pre if s["bias"] is None else pre + f(s["bias"])
        act = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0), "silu": lambda t: t * torch.sigmoid(t),
               "gelu": lambda t: t * torch.special.ndtr(t),
               "gelu_tanh": lambda t: t * torch.sigmoid((8 / math.pi) ** 0.5 * (t + 0.044715 * t ** 3))}[case["act"]](pre)
        if s["w_up"] is not None:
            up = torch.einsum("mk,nk->mn", f(s["x"]), f(s["w_up"]))
            act = act * (up if s["bias_up"] is None else up + f(s["bias_up"]))
        return act if s["residual"] is None else act + f(s["residual"])
    if case["kind"] == "norm":
        def standard(v, gain, bias):
            centre = v.mean(1) if case["norm"] == "layer" else torch.zeros_like(v[:, 0])
            spread = ((v - centre[:, None]) ** 2).mean(1)
            return (v - centre[:, None]) * torch.rsqrt(spread + 1e-5)[:, None] * f(gain) + (0 if bias is None else f(bias))
        t = f(s["y"]) if s["post_gain"] is None else standard(f(s["y"]), s["post_gain"], s["post_bias"])
        if s["gate"] is not None:
            g = f(s["gate"]).repeat_interleave(case["rows"] // s["gate"].shape[0], 0)
            t = t * (torch.tanh(g) if case["tanh"] else g)
        h = f(s["h"]) + case["scale"] * t
        return h, None if s["pre_gain"] is None else standard(h, s["pre_gain"], s["pre_bias"])
    heads, kv_heads, hd = MODELS[case["model"]][:3]
    group, window = heads // kv_heads, case["window"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for i, n in enumerate(_lens(case)):
        pages, rows = s["table"][i, : -(-n // PAGE)].long(), slice(i * window, (i + 1) * window)
        power = (s["exps"][pages, 0].long() + 1023 << 52).view(torch.float64).repeat_interleave(BLOCK, -1)   # 2^exponent
        k, v = ((s["pages"][pages, 0, j].double() * power[:, j, :, :, None]).transpose(0, 1).reshape(kv_heads, -1, hd)[:, :n] for j in (0, 1))
        a = torch.einsum("whgd,hnd->hgwn", f(s["q"][rows]).view(window, kv_heads, group, hd), k) * hd ** -0.5
        a = a.masked_fill(torch.arange(n, device="cuda") > s["in_pos"][rows].long()[:, None], -math.inf).softmax(-1)
        out[rows] = torch.einsum("hgwn,hnd->whgd", a, v).reshape(window, heads, hd)
    return out
