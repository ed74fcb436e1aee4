"""The operators around the 8-bit paged cache: what a call of each computes, in plain torch, and the cases that are timed.

  append     sjd_pool_append: rotary positions with several axes for q and k, k and v rounded to e4m3 with a power-of-two
             scale for each 16 positions and head, into the pages of a pool
  attention  sjd_pool_attention: window queries over those pages, causal, with an optional sliding window and sinks
  fork       sjd_pool_free + sjd_pool_fork + sjd_pool_reserve: children of a prompt share its pages, the partial last page
             is copied for the one that writes
  compact    sjd_pool_free + sjd_pool_compact + sjd_pool_reserve: a batch leaves, the pages that stay move down, a batch comes

A pool holds pages of 64 positions: bytes e4m3 [page][layer][K|V][kv_head][64][head_dim] and exponents int8
[page][layer][K|V][kv_head][4]; an entry stands for its e4m3 value times 2^exponent of its 16 positions.
Shapes follow the repository's own models: 32 heads of 128 with 32 or 8 kv heads, 8 heads of 64 with 2, windows of up to 64
(1063 for a prompt that holds an image), sequences of up to 128 + 4096 positions, and longer ones.
"""
import math

import torch

own = False

PAGE, BLOCK = 64, 16
HEADS = {"7b": (32, 32, 128), "8b-gqa": (32, 8, 128), "small": (8, 2, 64)}   # heads, kv heads, head_dim
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    att = dict(kind="attention", sliding=0, sinks=0, ragged=False)
    return [
        # the smallest call: one token of one short sequence of the small model
        dict(att, name="att_one_token", model="small", batch=1, window=1, length=217, dtype="bf16"),
        # a serving batch, a token each, sequences of different lengths
        dict(att, name="att_serve_b32", model="8b-gqa", batch=32, window=1, length=4224, dtype="bf16", ragged=True),
        # eight late images of the 7B decoder, windows of 32 drafts, fp32 activations
        dict(att, name="att_7b_late_b8", model="7b", batch=8, window=32, length=4009, dtype="f32"),
        # grouped heads with the widest window: 256 query rows share a kv head
        dict(att, name="att_gqa_w64", model="8b-gqa", batch=2, window=64, length=4224, dtype="bf16", ragged=True),
        # one very long sequence, few rows: the key axis has to be split
        dict(att, name="att_long", model="8b-gqa", batch=1, window=3, length=100003, dtype="bf16"),
        # a sliding window with a few first tokens that stay visible
        dict(att, name="att_sliding", model="8b-gqa", batch=4, window=32, length=20011, dtype="f32", sliding=1000, sinks=4, ragged=True),
        # every window of a batch of eight, fp32, image rows and columns as rotary axes
        dict(kind="append", name="append_window_b8", model="7b", batch=8, window=32, start=2311, dtype="f32", axes=3),
        # the prompt of one sequence
        dict(kind="append", name="append_prompt", model="8b-gqa", batch=1, window=4224, start=0, dtype="bf16", axes=1),
        # two children of a short prompt in a one-layer pool: launches and latency
        dict(kind="fork", name="fork_small", model="small", layers=1, children=2, length=100, write=16),
        # sixteen images of one prompt, all layers of a page
        dict(kind="fork", name="fork_16", model="8b-gqa", layers=32, children=16, length=1063, write=64),
        # a few pages move
        dict(kind="compact", name="compact_small", model="small", layers=2, batch=3, pages=5),
        # half of a pool moves
        dict(kind="compact", name="compact_large", model="8b-gqa", layers=32, batch=8, pages=40),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attention", "attention", "attention", "append", "append", "fork", "compact"))
    model = rng.choice(tuple(HEADS))
    heads, kv_heads, hd = HEADS[model]
    if kind == "attention":
        window = _log_int(rng, 1, 64) if rng.random() < 0.85 else _log_int(rng, 65, 1063)
        sliding = _log_int(rng, 1, 3000) if rng.random() < 0.4 else 0
        length = max(window, _log_int(rng, 1, 100003))
        if rng.random() < 0.6:
            length = max(window, min(length, 4224))
        batch = _log_int(rng, 1, 32)
        # no more keys times kv heads, and no more scores, than the largest listed case
        batch = max(1, min(batch, 8 * 32 * 4009 // (kv_heads * length), (1 << 25) // (heads * window * length)))
        length = max(window, min(length, (1 << 25) // (heads * window)))
        return dict(kind=kind, model=model, batch=batch, window=window, length=length, dtype=rng.choice(("f32", "bf16")),
                    sliding=sliding, sinks=_log_int(rng, 1, 128) if sliding and rng.random() < 0.6 else 0, ragged=rng.random() < 0.5)
    if kind == "append":
        batch = _log_int(rng, 1, 32)
        window = max(1, min(_log_int(rng, 1, 4224), 4224 // batch))
        return dict(kind=kind, model=model, batch=batch, window=window, start=rng.choice((0, _log_int(rng, 1, 4000))),
                    dtype=rng.choice(("f32", "bf16")), axes=rng.choice((1, 2, 3)))
    layers = _log_int(rng, 1, 32 if model != "7b" else 8)
    if kind == "fork":
        return dict(kind=kind, model=model, layers=layers, children=_log_int(rng, 1, 16), length=_log_int(rng, 1, 1063),
                    write=_log_int(rng, 1, 130))
    return dict(kind=kind, model=model, layers=layers, batch=_log_int(rng, 1, 8), pages=_log_int(rng, 1, 40))


# ---------------------------------------------------------------------------------------------------------------- states
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _page_bytes(n_pages, layers, kv_heads, hd, gen):
    """Random e4m3 entries as 16 normal rows fill them: a largest entry of 200 to 448."""
    x = torch.empty(n_pages, layers, 2, kv_heads, PAGE, hd, dtype=torch.float8_e4m3fn, device="cuda")
    for i in range(0, n_pages, 256):
        x[i:i + 256] = torch.randn(x[i:i + 256].shape, generator=gen, device="cuda").mul_(70).clamp_(-448, 448).to(torch.float8_e4m3fn)
    return x


def _pool(n_pages, n_seqs, per_seq, layers, kv_heads, hd, seed):
    gen = _gen(seed)
    s = {"pages": _page_bytes(n_pages, layers, kv_heads, hd, gen),
         "exps": torch.randint(-8, -5, (n_pages, layers, 2, kv_heads, PAGE // BLOCK), generator=gen, device="cuda").to(torch.int8),
         "table": torch.full((n_seqs, per_seq), -1, dtype=torch.int32, device="cuda"),
         "refs": torch.zeros(n_pages, dtype=torch.int32, device="cuda")}
    return s, gen


def _handle(s):
    """The framework's view of the pool, as a program that uses it keeps it."""
    if own:
        from paper_2410_01699_b200 import binding as B
        s["pool"] = B.CachePool(s["pages"], s["exps"], s["table"], s["refs"])
    return s


def _give_pages(s, counts, gen):
    """Sequence b gets counts[b] pages, in a random order of the pool's."""
    n = s["refs"].numel()
    order = torch.randperm(n, generator=gen, device="cuda").to(torch.int32)
    at = 0
    for b, c in enumerate(counts):
        s["table"][b, :c] = order[at:at + c]
        at += c
    s["refs"][order[:at].long()] = 1


def prepare(case, seed):
    heads, kv_heads, hd = HEADS[case["model"]]
    if case["kind"] == "attention":
        batch, window, length = case["batch"], case["window"], case["length"]
        lens = _lens(case)
        per_seq = -(-length // PAGE)
        counts = [-(-n // PAGE) for n in lens]
        s, gen = _pool(sum(counts) + 3, batch, per_seq, 1, kv_heads, hd, seed)
        _give_pages(s, counts, gen)
        s["exps"][s["table"][:, 0].long(), :, 1, :, 0] -= 3   # (values of first tokens are small)
        pos = torch.arange(window, device="cuda")[None] + torch.tensor(lens, device="cuda")[:, None] - window
        s["in_pos"] = pos.to(torch.int32).reshape(-1).contiguous()
        s["q"] = (torch.randn(batch * window, heads, hd, generator=gen, device="cuda") * 1.3).to(DTYPES[case["dtype"]])
        s["out"] = torch.empty_like(s["q"])
        s["table"].clamp_(min=0)
    elif case["kind"] == "append":
        batch, window, start = case["batch"], case["window"], case["start"]
        starts = [start - (b * 7) % (start // 2 + 1) for b in range(batch)]
        per_seq = -(-(start + window) // PAGE)
        s, gen = _pool(batch * per_seq + 1, batch, per_seq, 1, kv_heads, hd, seed)
        _give_pages(s, [per_seq] * batch, gen)
        # one matrix of queries, keys and values, as the projection leaves it
        qkv = torch.randn(batch * window, heads + 2 * kv_heads, hd, generator=gen, device="cuda")
        qkv[:, heads:] *= torch.exp(0.5 * torch.randn(batch * window, 2 * kv_heads, 1, generator=gen, device="cuda"))
        qkv = qkv.to(DTYPES[case["dtype"]])
        s["q"], s["k"], s["v"] = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        s["q_out"] = torch.empty(batch * window, heads, hd, dtype=qkv.dtype, device="cuda")
        pos = torch.arange(window, device="cuda")[None] + torch.tensor(starts, device="cuda")[:, None]
        s["in_pos"] = pos.to(torch.int32).reshape(-1).contiguous()
        p, half = s["in_pos"], hd // 2
        if case["axes"] == 1:
            s["axis_pos"], s["pairs"] = None, (half,)
        elif case["axes"] == 2:   # row and column of an image of 48 + 1 tokens a row
            s["axis_pos"], s["pairs"] = torch.stack((p // 49, p % 49), 1).contiguous(), (half // 2, half // 2)
        else:                     # time, height, width
            s["axis_pos"], s["pairs"] = torch.stack((p // 2401, p // 49 % 49, p % 49), 1).contiguous(), (half // 4, half * 3 // 8, half * 3 // 8)
    elif case["kind"] == "fork":
        n, length = case["children"], case["length"]
        per_seq = -(-(length + case["write"]) // PAGE)
        shared = -(-length // PAGE)
        s, gen = _pool(shared + n * (per_seq - shared + 1) + 1, n + 1, per_seq, case["layers"], kv_heads, hd, seed)
        _give_pages(s, [shared], gen)
        i32 = lambda v: torch.full((n,), v, dtype=torch.int32, device="cuda")
        s["children"] = torch.arange(1, n + 1, dtype=torch.int32, device="cuda")
        s["parent"], s["none"], s["len"], s["end"] = i32(0), i32(0), i32(length), i32(length + case["write"])
    else:
        n, pages = case["batch"], case["pages"]
        s, gen = _pool(2 * n * pages + 3, 2 * n, pages, case["layers"], kv_heads, hd, seed)
        _give_pages(s, [pages] * (2 * n), gen)
        i32 = lambda v: torch.full((n,), v, dtype=torch.int32, device="cuda")
        s["groups"] = [torch.arange(n, dtype=torch.int32, device="cuda") + g * n for g in range(2)]
        s["none"], s["end"], s["turn"] = i32(0), i32(pages * PAGE), 0
    s["case"] = dict(case)
    return _handle(s)


def _lens(case):
    length, window, batch = case["length"], case["window"], case["batch"]
    return [max(window, length - (b * length) // (2 * batch)) if case["ragged"] else length for b in range(batch)]


# ------------------------------------------------------------------------------------------------------------------ runs
def run(state):
    return {"attention": _attention, "append": _append, "fork": _fork, "compact": _compact}[state["case"]["kind"]](state)


def _attention(s):
    c = s["case"]
    if own:
        from paper_2410_01699_b200 import binding as B
        return B.sjd_pool_attention(s["pool"], 0, s["q"], s["in_pos"], c["window"], sliding=c["sliding"], sinks=c["sinks"], out=s["out"])
    m, heads, hd = s["q"].shape
    batch, window = m // c["window"], c["window"]
    kv_heads, per_seq = s["pages"].shape[3], s["table"].shape[1]
    at = s["table"].long()
    scale = torch.exp2(s["exps"][at][:, :, 0].float())                           # [b][page][K|V][kv head][block]
    kv = s["pages"][at][:, :, 0].float().view(batch, per_seq, 2, kv_heads, PAGE // BLOCK, BLOCK, hd) * scale[..., None, None]
    kv = kv.permute(2, 0, 3, 1, 4, 5, 6).reshape(2, batch, kv_heads, per_seq * PAGE, hd)
    q = s["q"].float().view(batch, window, kv_heads, heads // kv_heads, hd).permute(0, 2, 1, 3, 4).reshape(batch, kv_heads, -1, hd)
    score = torch.matmul(q, kv[0].transpose(-1, -2)) / math.sqrt(hd)
    pos = s["in_pos"].view(batch, 1, window, 1, 1)
    key = torch.arange(per_seq * PAGE, device="cuda")
    seen = key <= pos
    if c["sliding"]:
        seen = seen & ((key > pos - c["sliding"]) | (key < c["sinks"]))
    score = score.view(batch, kv_heads, window, -1, per_seq * PAGE).masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(batch, kv_heads, -1, per_seq * PAGE), kv[1]).view(batch, kv_heads, window, -1, hd)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return out.permute(0, 2, 1, 3, 4).reshape(m, heads, hd).to(s["q"].dtype)


def _append(s):
    c = s["case"]
    if own:
        from paper_2410_01699_b200 import binding as B
        B.sjd_pool_append(s["pool"], 0, s["k"], s["v"], s["in_pos"], c["window"], q=s["q"], q_out=s["q_out"],
                          rope=B.make_rope_cfg(s["pairs"]), axis_pos=s["axis_pos"])
        return {"q": s["q_out"], "cache": s["pages"], "exponents": s["exps"]}
    hd = s["q"].shape[-1]
    half, window, batch = hd // 2, c["window"], c["batch"]
    # angles in 64 bits, their cosine and sine rounded to 32
    pair = torch.arange(half, device="cuda")
    freq = 10000.0 ** (-2.0 * pair.double() / hd)
    axis = torch.repeat_interleave(torch.arange(len(s["pairs"]), device="cuda"), torch.tensor(s["pairs"], device="cuda"))
    pos = s["in_pos"][:, None].expand(-1, half) if s["axis_pos"] is None else s["axis_pos"][:, axis]
    angle = pos.double() * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotate(x):
        a, b = x[..., :half].float(), x[..., half:].float()
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)

    s["q_out"].copy_(rotate(s["q"]))
    new = torch.stack((rotate(s["k"]), s["v"].float()), 1).view(batch, window, 2, -1, hd)
    # the blocks of 16 positions that the window touches: what stays of them, and the new rows
    first = s["in_pos"].view(batch, window)[:, :1].long()
    begin = first // BLOCK * BLOCK
    n = (window + BLOCK - 2) // BLOCK + 1
    at = begin + torch.arange(n * BLOCK, device="cuda")                          # [b][row]: positions
    inside = at < first + window
    logical = (at // PAGE).clamp(max=s["table"].shape[1] - 1)
    page, row = s["table"].gather(1, logical).long(), at % PAGE
    old = s["pages"].view(torch.uint8)[page, 0, :, :, row].view(torch.float8_e4m3fn).float()   # [b][row][K|V][kv head][hd]
    old = old * torch.exp2(s["exps"][page, 0, :, :, row // BLOCK].float())[..., None]
    k = (at - first).clamp(0, window - 1)
    rows = torch.where((at < first)[..., None, None, None], old, new[torch.arange(batch, device="cuda")[:, None], k])
    rows = torch.where(inside[..., None, None, None], rows, torch.zeros_like(rows)).view(batch, n, BLOCK, 2, -1, hd)
    # the smallest power of two that holds the block's largest entry in 448 (0 where all are zero)
    top = rows.abs().amax((2, 5))                                                # [b][block][K|V][kv head]
    frac, e = torch.frexp(top)
    e = torch.where(top > 0, e - 9 + (frac > 0.875), torch.zeros_like(e)).clamp(-100, 100)
    byte = (rows * torch.exp2(-e.float())[:, :, None, :, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    byte = byte.view(batch, n * BLOCK, 2, -1, hd)
    b, r = torch.nonzero(inside, as_tuple=True)
    s["pages"].view(torch.uint8)[page[b, r], 0, :, :, row[b, r]] = byte[b, r]
    b, r = torch.nonzero(inside.view(batch, n, BLOCK)[:, :, 0], as_tuple=True)
    s["exps"][page[b, r * BLOCK], 0, :, :, row[b, r * BLOCK] // BLOCK] = e[b, r].to(torch.int8)
    return {"q": s["q_out"], "cache": s["pages"], "exponents": s["exps"]}


def _plain_free(s, seqs, keep):
    table = s["table"][seqs.long()]
    gone = (torch.arange(table.shape[1], device="cuda") >= (keep[:, None] + PAGE - 1) // PAGE) & (table >= 0)
    s["refs"].index_add_(0, table[gone].long(), torch.full_like(table[gone], -1))
    s["table"][seqs.long()] = torch.where(gone, -1, table)


def _plain_fork(s, src, dst, length):
    table = s["table"][src.long()]
    kept = torch.arange(table.shape[1], device="cuda") < (length[:, None] + PAGE - 1) // PAGE
    s["table"][dst.long()] = torch.where(kept, table, -1)
    s["refs"].index_add_(0, table[kept].long(), torch.ones_like(table[kept]))


def _plain_reserve(s, seqs, begin, end):
    """Pages for positions begin .. end - 1: absent ones are given, shared ones are replaced (but by their last holder)."""
    table = s["table"][seqs.long()]
    i = torch.arange(table.shape[1], device="cuda")
    wanted = (i >= begin[:, None] // PAGE) & (i * PAGE < end[:, None])
    row, col = torch.nonzero(wanted, as_tuple=True)
    page = table[row, col].long()
    have = page >= 0
    # how many of this call's earlier claims are for the same page
    order = torch.arange(page.numel(), device="cuda")
    by_page = torch.argsort(torch.where(have, page, s["refs"].numel() + order), stable=True)
    sorted_page = page[by_page]
    run_start = torch.cummax(torch.where(torch.cat((by_page.new_ones(1, dtype=torch.bool), sorted_page[1:] != sorted_page[:-1])),
                                         order, torch.zeros_like(order)), 0)[0]
    earlier = torch.empty_like(order)
    earlier[by_page] = order - run_start
    shared = have & (s["refs"][page.clamp(min=0)] - earlier > 1)
    new = ~have | shared
    got = torch.nonzero(s["refs"] == 0)[:, 0][: int(new.sum())]
    row, col, page, copied = row[new], col[new], page[new], (shared & (col * PAGE < begin[row]))[new]
    s["pages"].view(torch.uint8)[got[copied]] = s["pages"].view(torch.uint8)[page[copied]]
    s["exps"][got[copied]] = s["exps"][page[copied]]
    s["refs"].index_add_(0, page[page >= 0], torch.full_like(page[page >= 0], -1, dtype=torch.int32))
    s["refs"][got] = 1
    s["table"][seqs.long()[row], col] = got.to(torch.int32)


def _plain_compact(s):
    live = s["refs"] > 0
    n = int(live.sum())
    index = torch.arange(live.numel(), device="cuda")
    src, dst = index[live & (index >= n)], index[~live & (index < n)]
    s["pages"].view(torch.uint8)[dst] = s["pages"].view(torch.uint8)[src]
    s["exps"][dst] = s["exps"][src]
    s["refs"][dst] = s["refs"][src]
    s["refs"][src] = 0
    to = index.to(torch.int32)
    to[src] = dst.to(torch.int32)
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], s["table"]))


def _state(s):
    return {"cache": s["pages"], "exponents": s["exps"], "table": s["table"], "refs": s["refs"]}


def _fork(s):
    """The children of the last pass go, new ones come and make room for what they write next."""
    if own:
        from paper_2410_01699_b200 import binding as B
        B.sjd_pool_free(s["pool"], s["children"], s["none"])
        B.sjd_pool_fork(s["pool"], s["parent"], s["children"], s["len"])
        B.sjd_pool_reserve(s["pool"], s["children"], s["len"], s["end"])
        return _state(s)
    _plain_free(s, s["children"], s["none"])
    _plain_fork(s, s["parent"], s["children"], s["len"])
    _plain_reserve(s, s["children"], s["len"], s["end"])
    return _state(s)


def _compact(s):
    """One half of the sequences goes, the pages of the other half move down, the first half comes again."""
    go = s["groups"][s["turn"]]
    s["turn"] ^= 1
    if own:
        from paper_2410_01699_b200 import binding as B
        B.sjd_pool_free(s["pool"], go, s["none"])
        B.sjd_pool_compact(s["pool"])
        B.sjd_pool_reserve(s["pool"], go, s["none"], s["end"])
        return _state(s)
    _plain_free(s, go, s["none"])
    _plain_compact(s)
    _plain_reserve(s, go, s["none"], s["end"])
    return _state(s)


# ------------------------------------------------------------------------------------------------------------------ work
def work(case):
    heads, kv_heads, hd = HEADS[case["model"]]
    page = case.get("layers", 1) * 2 * kv_heads * (PAGE * hd + PAGE // BLOCK)
    if case["kind"] == "attention":
        size, window = DTYPES[case["dtype"]].itemsize, case["window"]
        keys = pairs = 0
        for n in _lens(case):
            if case["sliding"]:
                # (the rows' windows overlap: one range, and the sinks before it)
                low = max(0, n - window + 1 - case["sliding"])
                keys += n - low + min(low, case["sinks"])
                pairs += sum(min(p + 1, case["sliding"]) + min(max(0, p + 1 - case["sliding"]), case["sinks"]) for p in range(n - window, n))
            else:
                keys += n
                pairs += sum(range(n - window + 1, n + 1))
        rows = case["batch"] * window
        return {"bytes": keys * 2 * kv_heads * hd * (1 + 1 / (BLOCK * hd)) + 2 * rows * heads * hd * size + rows * 4,
                "flops": 4.0 * hd * heads * pairs}
    if case["kind"] == "append":
        rows, size = case["batch"] * case["window"], DTYPES[case["dtype"]].itemsize
        return {"bytes": rows * hd * (2 * heads * size + 2 * kv_heads * (size + 1)), "flops": rows * hd * (3 * heads + 5 * kv_heads)}
    if case["kind"] == "fork":
        # the partial page is read once and written once for each child; tables and counts
        n, copied = case["children"], case["length"] % PAGE != 0
        per_seq = -(-(case["length"] + case["write"]) // PAGE)
        return {"bytes": (1 + n) * page * copied + n * per_seq * 16, "flops": 0}
    n = case["batch"] * case["pages"]
    # a page that moves is read and written: the pages of the staying half that lie behind its count (about half of them)
    return {"bytes": 2 * page * max(1, n // 2) + n * 24, "flops": 0}


# ----------------------------------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The definition in 64 bits, one sequence (and kv head) at a time.  The page operations move whole numbers and bytes: no
    value of theirs is computed."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "attention":
        return _exact_attention(case, s)
    if case["kind"] == "append":
        return _exact_append(case, s)
    return None


def _exact_attention(case, s):
    m, heads, hd = s["q"].shape
    kv_heads, window = s["pages"].shape[3], case["window"]
    group = heads // kv_heads
    out = torch.zeros(m, heads, hd, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(case)):
        pages = s["table"][b, : -(-n // PAGE)].long()
        for h in range(kv_heads):
            k, v = ((s["pages"][pages, 0, j, h].double().view(-1, BLOCK, hd) * _two_to(s["exps"][pages, 0, j, h]).view(-1, 1, 1))
                    .view(-1, hd)[:n] for j in range(2))
            q = s["q"][b * window:(b + 1) * window, h * group:(h + 1) * group].double()
            a = torch.einsum("wgd,nd->wgn", q, k) * hd ** -0.5
            far = (s["in_pos"][b * window:(b + 1) * window].long()[:, None] - torch.arange(n, device="cuda"))[:, None]
            hidden = far < 0
            if case["sliding"]:
                hidden = hidden | ((far >= case["sliding"]) & (torch.arange(n, device="cuda") >= case["sinks"]))
            a = a.masked_fill(hidden, -math.inf).softmax(-1)
            out[b * window:(b + 1) * window, h * group:(h + 1) * group] = torch.einsum("wgn,nd->wgd", a, v)
    return out


def _two_to(e):
    """2^e in 64 bits to the last one, which a power function does not promise."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _round_e4m3(x):
    """Nearest multiple of the step of x's binade (2^-9 at least), ties to the even one."""
    step = _two_to(torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(x / step) * step


def _exact_append(case, s):
    heads, kv_heads, hd = HEADS[case["model"]]
    half, window = hd // 2, case["window"]
    axis = sum(([a] * n for a, n in enumerate(s["pairs"])), [])
    q, cache = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), s["pages"].double()
    exps = s["exps"].clone()
    for b in range(case["batch"]):
        at = slice(b * window, (b + 1) * window)
        pos = (s["in_pos"][at, None] if s["axis_pos"] is None else s["axis_pos"][at]).double()
        turn = torch.stack([pos[:, a] * 10000.0 ** (-i / half) for i, a in enumerate(axis)], 1)
        turn = torch.polar(torch.ones_like(turn), turn)[:, None]
        spin = lambda x: (lambda z: torch.cat((z.real, z.imag), -1))(torch.complex(x[..., :half].double(), x[..., half:].double()) * turn)
        q[at] = spin(s["q"][at])
        new = torch.stack((spin(s["k"][at]), s["v"][at].double()))                       # [K|V][row][kv head][hd]
        p0 = int(s["in_pos"][b * window])
        for base in range(p0 // BLOCK * BLOCK, p0 + window, BLOCK):
            page, block = int(s["table"][b, base // PAGE]), base % PAGE // BLOCK
            rows = slice(block * BLOCK, block * BLOCK + min(BLOCK, p0 + window - base))
            kept = max(0, p0 - base)
            old = cache[page, 0, :, :, block * BLOCK:block * BLOCK + kept] * _two_to(exps[page, 0, :, :, block])[..., None, None]
            now = torch.cat((old, new[:, base + kept - p0:base + BLOCK - p0].transpose(1, 2)), 2)
            top = now.abs().amax((2, 3))
            e = torch.round(torch.log2(top.clamp(min=1e-300) / 448))   # (a logarithm next to a whole number may be on either side of it)
            e = torch.where(top > 448 * _two_to(e), e + 1, e).clamp(-100, 100) * (top > 0)
            cache[page, 0, :, :, rows] = _round_e4m3((now / _two_to(e)[..., None, None]).clamp(-448, 448))
            exps[page, 0, :, :, block] = e.to(torch.int8)
    return {"q": q, "cache": cache, "exponents": exps}
