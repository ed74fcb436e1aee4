"""sjd_pool_attention_shared: refusals without a GPU; on one against oracle/pool.py, which knows nothing of shared pages."""
import ctypes as C
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from oracle import pool as O
from paper_2410_01699_b200 import binding as B

FAKE = 1 << 20   # an address that no refused call may use


def _call(pool=None, **kw):
    f = dict(pages=FAKE, exps=FAKE, table=FAKE, refs=FAKE, status=FAKE, n_pages=8, n_seqs=4, pages_per_seq=4, n_layers=2, n_kv_heads=2, head_dim=64)
    f.update(pool or {})
    p = B.sjd_pool(*[f[n] for n, _ in B.sjd_pool._fields_])
    a = dict(layer=0, batch=4, window=4, heads=4, dtype=1, q=FAKE, qs=256, seqs=None, in_pos=FAKE, n_groups=1, groups=None, scale=0.0, out=FAKE,
             outs=256, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return B.lib().sjd_pool_attention_shared(C.byref(p), *a.values(), None)


@pytest.mark.parametrize("change,status", [
    (dict(pool=dict(pages=None)), B.SJD_ERR_BAD_ARG), (dict(pool=dict(head_dim=96)), B.SJD_ERR_UNSUPPORTED), (dict(dtype=0), B.SJD_ERR_UNSUPPORTED),
    (dict(layer=2), B.SJD_ERR_BAD_ARG), (dict(layer=-1), B.SJD_ERR_BAD_ARG), (dict(batch=0), B.SJD_ERR_BAD_ARG), (dict(window=0), B.SJD_ERR_BAD_ARG),
    (dict(heads=3), B.SJD_ERR_BAD_ARG), (dict(q=None), B.SJD_ERR_BAD_ARG), (dict(in_pos=None), B.SJD_ERR_BAD_ARG), (dict(out=None), B.SJD_ERR_BAD_ARG),
    (dict(ws=None), B.SJD_ERR_BAD_ARG), (dict(ws=FAKE + 128), B.SJD_ERR_BAD_ARG), (dict(qs=252), B.SJD_ERR_BAD_ARG), (dict(outs=258), B.SJD_ERR_BAD_ARG),
    (dict(q=FAKE + 4), B.SJD_ERR_BAD_ARG), (dict(out=FAKE + 4), B.SJD_ERR_BAD_ARG), (dict(scale=-1.0), B.SJD_ERR_BAD_ARG),
    (dict(scale=float("nan")), B.SJD_ERR_BAD_ARG), (dict(groups=FAKE, n_groups=0), B.SJD_ERR_BAD_ARG), (dict(groups=FAKE + 2), B.SJD_ERR_BAD_ARG),
    (dict(seqs=FAKE + 1), B.SJD_ERR_BAD_ARG), (dict(groups=FAKE, n_groups=5), B.SJD_ERR_CAPACITY), (dict(batch=1025), B.SJD_ERR_CAPACITY),
    (dict(ws_bytes=1 << 10), B.SJD_ERR_CAPACITY), (dict(pool=dict(pages_per_seq=1 << 20, n_seqs=1 << 10), batch=1024, window=1000, ws_bytes=1 << 45), B.SJD_ERR_CAPACITY)])
def test_refusals(change, status):
    assert _call(**change) == status


def test_workspace_size_query():
    pool = B.sjd_pool(FAKE, FAKE, FAKE, FAKE, FAKE, 8, 4, 4, 2, 2, 64)
    size = lambda *a: int(B.lib().sjd_pool_attention_shared_workspace_bytes(C.byref(pool), *a))
    assert 0 < size(1, 1, 2) <= size(4, 16, 4) < size(4, 64, 16)
    assert size(0, 1, 2) == size(1, 0, 2) == size(1, 1, 3) == size(1025, 1, 2) == size(1024, 1 << 20, 2) == 0


def test_workspaces_of_a_pool_whose_calls_grow():
    """Those that were too small stay, for graphs that hold them, but do not add up."""
    pool = B.CachePool.empty(4, 2, 4, 1, 2, 64, device="cpu")
    need, kept = [], []
    for batch in range(1, 400):
        need.append(int(B.lib().sjd_pool_attention_shared_workspace_bytes(pool.ref, batch, 40, 16)))
        ws = pool.shared_ws(batch, 40, 16)
        kept += [ws] if not kept or ws is not kept[-1] else []
        assert ws.nbytes >= need[-1]
    assert need[-1] > 2 * need[0] and len(kept) <= 4 and all(a is b for a, b in zip(pool._shared_ws, kept))
    assert sum(x.nbytes for x in pool._shared_ws) < 4 * need[-1]
    assert pool.shared_ws(1, 40, 16) is kept[-1] and pool.shared_ws(399, 40, 16) is kept[-1]


# ------------------------------------------------------------------------------------------- which kernel a call comes to
def _each_for_itself(calls):
    """The library's rule (csrc/pool_route.h) for calls (batch, window, kv_heads, rows, pages_per_seq, alone, sms)."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "route.cpp"), os.path.join(d, "route")
        with open(src, "w") as f:
            f.write('#include <cstdio>\n#include "pool_route.h"\nint main() {\n  long a[7];\n'
                    '  while (std::scanf("%ld %ld %ld %ld %ld %ld %ld", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6) == 7)\n'
                    '    std::printf("%d\\n", (int)sjd::pool_each_for_itself(a[0], a[1], a[2], a[3], a[4], a[5], a[6]));\n}\n')
        subprocess.run(["g++", "-std=c++17", "-I" + os.path.join(root, "include"),
                        "-I" + os.path.join(root, "paper_2410_01699_b200", "csrc"), src, "-o", exe], check=True)
        text = "".join(" ".join(str(int(x)) for x in c) + "\n" for c in calls)
        return [bool(int(x)) for x in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()]


def test_short_and_lone_calls_are_left_to_attention_of_every_sequence():
    assert _each_for_itself([(2, 1, 4, 1, 4, 0, 148), (2, 1, 32, 1, 100, 0, 148), (32, 16, 32, 16, 34, 0, 148), (64, 1, 8, 4, 516, 0, 148),      # by what the tables hold
                             (32, 1, 8, 4, 1 << 20, 1, 148), (16, 16, 8, 64, 1 << 20, 1, 148), (16, 32, 8, 128, 1 << 20, 1, 148),                # nobody can share
                             (600, 1, 1, 1, 2, 0, 148), (1024, 1, 8, 4, 4, 1, 148), (9, 1000, 1, 1000, 16, 0, 148)]) == \
        [True, True, False, False, True, True, False, False, False, False]


# ------------------------------------------------------------------------------------------------------------------ values
LONG = 16384   # pages of a sequence's table: a call with such tables is not left to sjd_pool_attention for its length


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _filled(groups, n_layers, kvh, hd, seed, spare=3, exps=(-8, -5), per_seq=LONG):
    """A pool and the lengths of its sequences.  groups: (shared pages, lengths); pages in random order; rows behind a sequence hold anything."""
    rng = np.random.default_rng(seed)
    lens = [n for _, of in groups for n in of]
    shared = [k for k, of in groups for _ in of]
    n = sum(k for k, _ in groups) + sum(-(-x // 64) - min(k, -(-x // 64)) for x, k in zip(lens, shared)) + spare
    gen = torch.Generator().manual_seed(seed)
    pages = (torch.randn(n, n_layers, 2, kvh, 64, hd, generator=gen) * 70).clamp(-448, 448).to(torch.float8_e4m3fn)
    table = np.full((len(lens), max([per_seq] + [-(-x // 64) for x in lens])), -1, np.int32)
    order, at, refs, b = rng.permutation(n), 0, np.zeros(n, np.int32), 0
    for k, of in groups:
        common = order[at:at + k]
        at += k
        for x in of:
            have = -(-x // 64)
            table[b, :min(k, have)] = common[:have]
            own = have - min(k, have)
            table[b, k:k + own] = order[at:at + own]
            at += own
            refs[table[b, :have]] += 1
            if x % 64 and have > k:
                tail = pages.view(torch.uint8)[table[b, have - 1], ..., x % 64:, :]
                tail.copy_(torch.from_numpy(rng.integers(0, 256, tail.shape, dtype=np.uint8)))
                tail[..., ::3] = 0x7F
            b += 1
    ex = torch.from_numpy(rng.integers(exps[0], exps[1] + 1, (n, n_layers, 2, kvh, 4)).astype(np.int8))
    return B.CachePool(pages.cuda(), ex.cuda(), torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda()), lens


def _begin(groups):
    return _i32(np.cumsum([0] + [len(of) for _, of in groups]).tolist())


def _oracle(pool):
    return O.Pool(pool.pages.view(torch.uint8).cpu().numpy(), pool.exps.cpu().numpy(), pool.table.cpu().numpy(), pool.refs.cpu().numpy())


def _window_pos(lens, window, active=None):
    out = []
    for b, n in enumerate(lens):
        k = min(n, window if active is None else active[b])
        out += [n - k + i for i in range(k)] + [-1] * (window - k)
    return out


def _queries(m, heads, hd, seed, spread=1.3):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(m, heads, hd, generator=g) * spread).bfloat16().cuda()


def _bound(want, n):
    """Most that an output may be off.  A weight is rounded to bf16: 2^-8 of itself.  A query's two e4m3 numbers hold the eight bits of its entries but
    for half of the smallest step, 2^-10 where the row's largest is 2^7 or more (flat).  Products are exact; tensor memory adds some of them a
    step and rounds towards zero, up to eight steps, and the products with the factors, the reference and the exponential's argument are rounded:
    2^-19 of a score's magnitudes (reach) covers them; a score counts twice, in the numerator and in the sum.  The sums over n keys: n / 16 steps of 2^-23, factors and joints of
    parts 2^-15.  The output's own rounding: half a step, 2^-8."""
    out, mass, _, reach, flat = want
    score = reach * 2.0 ** -19 + flat * 2.0 ** -17
    return 1.02 * ((2.0 ** -8 + 2 * score[..., None] + 2.0 ** -15 + n / 16 * 2.0 ** -23) * mass) + 2.0 ** -8 * np.abs(out) + 1e-35


def _check(pool, q, in_pos, window, begin, scale=0.0, seqs=None, layer=0, out=None):
    """Results within their bounds.  Calls that are left to sjd_pool_attention (all are asked for with tables as short as they can be, too) are its results."""
    batch = len(in_pos) // window
    at, of = _i32(in_pos), _i32(seqs) if seqs is not None else None
    each = B.sjd_pool_attention(pool, layer, q, at, window, scale=scale, seqs=of)
    short = B.CachePool(pool.pages, pool.exps, pool.table[:, :max(max(in_pos), 0) // 64 + 1].contiguous(), pool.refs)
    got = B.sjd_pool_attention_shared(short, layer, q, at, window, group_begin=begin, scale=scale, seqs=of)
    assert short.fault() == 0
    if not torch.equal(got, B.sjd_pool_attention(short, layer, q, at, window, scale=scale, seqs=of)):   # (which cuts long tables otherwise)
        _within(pool, got, q, in_pos, window, scale, seqs, layer)
    if batch == 1 and window * q.shape[1] // pool.pages.shape[3] <= 64:
        out = B.sjd_pool_attention_shared(pool, layer, q, at, window, group_begin=begin, scale=scale, seqs=of, out=out)
        assert torch.equal(out, each) and pool.fault() == 0
        return out
    if begin is not None and begin.numel() == batch + 1:   # (all alone: as one group they come to the kernel)
        got = B.sjd_pool_attention_shared(pool, layer, q, at, window, group_begin=begin, scale=scale, seqs=of)
        if not torch.equal(got, each):
            _within(pool, got, q, in_pos, window, scale, seqs, layer)
        begin = None
    out = B.sjd_pool_attention_shared(pool, layer, q, at, window, group_begin=begin, scale=scale, seqs=of, out=out)
    assert pool.fault() == 0
    _within(pool, out, q, in_pos, window, scale, seqs, layer)
    return out


def _within(pool, out, q, in_pos, window, scale=0.0, seqs=None, layer=0):
    batch = len(in_pos) // window
    exact = _oracle(pool).attention(layer, q.float().cpu().numpy(), seqs if seqs is not None else range(batch), in_pos, window, 0, 0, scale)
    got = out.float().cpu().numpy().astype(np.float64)
    err, tol = np.abs(got - exact[0]), _bound(exact, max(in_pos) + 1)
    assert np.isfinite(got).all()
    assert (err <= tol).all(), "worst %.3g of its bound at %s" % ((err / tol).max(), np.unravel_index((err / tol).argmax(), err.shape))
    for m, at in enumerate(in_pos):
        assert at >= 0 or (got[m] == 0).all()
    norm = np.linalg.norm(exact[0])
    assert norm == 0 or np.linalg.norm(got - exact[0]) / norm <= 2.0 ** -8


HEADS = [(4, 2, 64), (4, 1, 128), (3, 3, 128), (6, 1, 64), (8, 2, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kvh,hd", HEADS)
@pytest.mark.parametrize("groups", [[(0, [1])], [(0, [64, 65])], [(1, [65, 66])], [(2, [128, 129])], [(2, [130, 200, 129])], [(3, [193, 500]), (2, [150, 140, 300])],
                                    [(5, [321] * 7)], [(4, [257]), (0, [3, 70]), (4, [300, 301])]])
def test_single_tokens(heads, kvh, hd, groups):
    pool, lens = _filled(groups, 1, kvh, hd, 1)
    _check(pool, _queries(len(lens), heads, hd, 2), _window_pos(lens, 1), 1, _begin(groups))


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kvh,hd", HEADS)
@pytest.mark.parametrize("window,groups", [(2, [(2, [150, 160])]), (16, [(3, [210, 230, 301])]), (17, [(2, [145, 300]), (5, [340, 700, 337])]), (33, [(4, [289, 290, 300, 310])]),
                                           (64, [(2, [192, 500, 193])]), (100, [(3, [300, 340])]), (300, [(1, [400, 364]), (2, [430, 428])])])
def test_windows(heads, kvh, hd, window, groups):
    pool, lens = _filled(groups, 1, kvh, hd, 3)
    _check(pool, _queries(len(lens) * window, heads, hd, 4), _window_pos(lens, window), window, _begin(groups))


@pytest.mark.gpu
def test_without_groups_all_are_one():
    groups = [(3, [200, 260, 300])]
    pool, lens = _filled(groups, 2, 2, 64, 5)
    q = _queries(3 * 4, 4, 64, 6)
    a = _check(pool, q, _window_pos(lens, 4), 4, None, layer=1)
    assert torch.equal(a, _check(pool, q, _window_pos(lens, 4), 4, _begin(groups), layer=1))
    _check(pool, q, _window_pos(lens, 4), 4, _i32([0, 1, 2, 3]))   # (nobody shares)
    _check(pool, q, _window_pos(lens, 4), 4, _i32([0, 0, 2, 3]), scale=0.3)   # (a group of none)


@pytest.mark.gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_sequences_of_a_group_that_share_less_or_nothing(hd):
    """Tables part at another page each; rows that are still within the common pages; a sequence twice."""
    pool, lens = _filled([(6, [400, 420, 500, 450])], 1, 1, hd, 7, spare=20)
    own = torch.nonzero(pool.refs == 0)[:6, 0].to(torch.int32)
    pool.table[1, 4:6] = own[:2]      # (pages with other contents)
    pool.table[3, 2:6] = own[2:6]
    q = _queries(4 * 8, 4, hd, 8)
    for order in ([0, 1, 2, 3], [3, 2, 1, 0], [0, 2, 0, 2], [1, 1, 1, 1]):
        _check(pool, q, _window_pos([lens[i] for i in order], 8), 8, None, seqs=order)
        _check(pool, q, _window_pos([lens[i] for i in order], 8), 8, _i32([0, 2, 4]), seqs=order)
    pos = _window_pos([lens[i] for i in (0, 2, 0, 2)], 8)
    pos[3] = 200                      # (the common pages end before this row)
    _check(pool, q, pos, 8, None, seqs=[0, 2, 0, 2])
    pos[9] = 0
    _check(pool, q, pos, 8, None, seqs=[0, 2, 0, 2])


@pytest.mark.gpu
@pytest.mark.parametrize("least", [3, 40])
def test_many_sequences_that_part_at_pages_of_their_own(least):
    """Hundreds of a group, more than warps that compare their tables: what they share is lowered by many at a time.  Nothing depends on which comes first."""
    groups = [(44, [44 * 64 + 1 + 7 * i % 90 for i in range(300)]), (44, [44 * 64 + 3 + 5 * i % 70 for i in range(40)])]
    pool, lens = _filled(groups, 1, 1, 64, 53, spare=700)
    rng, own = np.random.default_rng(54), torch.nonzero(pool.refs == 0)[:, 0].to(torch.int32)
    where = rng.integers(least, 44, len(lens))
    where[0], where[-1] = 43, least
    pool.table[torch.arange(len(lens)), torch.from_numpy(where)] = own[:len(lens)]   # (pages with other contents)
    q, at = _queries(len(lens), 2, 64, 55), _window_pos(lens, 1)
    a = _check(pool, q, at, 1, _begin(groups))
    for _ in range(10):
        assert torch.equal(a, B.sjd_pool_attention_shared(pool, 0, q, _i32(at), 1, group_begin=_begin(groups)))
    assert pool.fault() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kvh,hd,window", [(2, 1, 128, 9), (4, 4, 64, 40), (8, 1, 128, 40)])
def test_rows_and_sequences_that_see_nothing(heads, kvh, hd, window):
    groups = [(3, [200, 260, 300, 250]), (2, [150, 0, 170]), (0, [0, 0])]
    pool, lens = _filled(groups, 1, kvh, hd, 9)
    active = (window, 1, 0, 5, window, 0, 3, 0, 0)
    out = torch.full((len(lens) * window, heads, hd), 7.0, device="cuda").bfloat16()
    _check(pool, _queries(len(lens) * window, heads, hd, 10), _window_pos(lens, window, active), window, _begin(groups), out=out)
    out = B.sjd_pool_attention_shared(pool, 0, _queries(4, heads, hd, 4), _i32([-1] * 4), 1)
    assert (out == 0).all() and pool.fault() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("window,heads,kvh,hd,groups", [(1, 4, 1, 128, [(300, [19300, 19201, 19500])]), (3, 8, 2, 64, [(100, [6500, 9000]), (50, [3300, 3250, 3204])]),
                                                       (64, 4, 1, 128, [(40, [2700, 2625, 2800, 3000, 2624])]), (32, 2, 2, 128, [(30, [2000] * 5), (0, [4009])])])
def test_long_sequences_are_spread_over_the_device(window, heads, kvh, hd, groups):
    pool, lens = _filled(groups, 1, kvh, hd, 11)
    q, at, begin = _queries(len(lens) * window, heads, hd, 12), _window_pos(lens, window), _begin(groups)
    a = _check(pool, q, at, window, begin)
    for _ in range(3):   # the workspace is ready again, and nothing depends on the order of arrival
        assert torch.equal(a, B.sjd_pool_attention_shared(pool, 0, q, _i32(at), window, group_begin=begin))


@pytest.mark.gpu
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window,groups", [(1, [(5, [400, 390])]), (8, [(9, [700, 641])]), (8, [(9, [700, 641]), (2, [300, 290])]), (16, [(20, [1400, 1390])])])
def test_units_whose_rows_both_streams_have(hd, window, groups):
    """Up to 128 rows: every other tile is a stream's, and each reads the sums of both.  (The last case has more rows: beside them.)"""
    pool, lens = _filled(groups, 1, 2, hd, 56)
    q, at, begin = _queries(len(lens) * window, 16, hd, 57), _window_pos(lens, window), _begin(groups)
    a = _check(pool, q, at, window, begin)
    for _ in range(20):
        assert torch.equal(a, B.sjd_pool_attention_shared(pool, 0, q, _i32(at), window, group_begin=begin))


@pytest.mark.gpu
def test_many_sequences():
    """1024 sequences in groups of 1 to 40, more units than places kept in shared memory."""
    rng, groups, left = np.random.default_rng(13), [], 1024
    while left:
        n, k = min(left, int(rng.integers(1, 41))), int(rng.integers(0, 5))
        groups.append((k, (k * 64 + rng.integers(1, 150, n)).tolist()))
        left -= n
    pool, lens = _filled(groups, 1, 1, 64, 14)
    _check(pool, _queries(1024, 2, 64, 15), _window_pos(lens, 1), 1, _begin(groups))
    # and windows whose rows are more than a tile's: 3 tiles each
    pool, lens = _filled([(0, [150] * 800)], 1, 1, 64, 16)
    window, rows = 150, [0, 1, 149, 150, 5000, 77777, 119998, 119999]
    q, at = _queries(800 * window, 4, 64, 17), _window_pos(lens, window)
    got = B.sjd_pool_attention_shared(pool, 0, q, _i32(at), window).float().cpu().numpy()
    ref = _oracle(pool)
    for m in rows:
        want = ref.attention(0, q[m:m + 1].float().cpu().numpy(), [m // window], [at[m]], 1)
        assert (np.abs(got[m] - want[0][0]) <= _bound(want, 150)[0]).all()
    assert pool.fault() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kvh,hd,window", [(2, 1, 64, 5), (2, 1, 128, 5), (8, 1, 128, 30), (8, 2, 64, 40)])
def test_a_nan_shows_where_it_is_seen_and_nowhere_else(heads, kvh, hd, window):
    groups = [(3, [300, 260, 285])]
    pool, lens = _filled(groups, 1, kvh, hd, 18)
    q, at = _queries(3 * window, heads, hd, 19), _window_pos(lens, window)
    clean = _check(pool, q, at, window, _begin(groups)).float().cpu().numpy()
    raw, table = pool.pages.view(torch.uint8), pool.table.cpu().numpy()
    for b, key, dim in ((0, 100, 5), (1, 258, 7), (2, 283, hd - 1), (2, 284, 0)):   # one among the shared pages, others that some rows see
        kept = raw[table[b, key // 64], 0, 1, 0, key % 64, dim].item()
        raw[table[b, key // 64], 0, 1, 0, key % 64, dim] = 0xFF
        got = B.sjd_pool_attention_shared(pool, 0, q, _i32(at), window, group_begin=_begin(groups)).float().cpu().numpy()
        for m, p in enumerate(at):
            bad = np.isnan(got[m])
            if key < 192 or (m // window == b and p >= key):
                assert bad[:heads // kvh, dim].all() and bad.sum() == heads // kvh
            else:
                assert not bad.any()
            assert np.array_equal(got[m][~bad], clean[m][~bad])
        raw[table[b, key // 64], 0, 1, 0, key % 64, dim] = kept
    kept = raw[table[1, 258 // 64], 0, 0, 0, 258 % 64, 3].item()
    raw[table[1, 258 // 64], 0, 0, 0, 258 % 64, 3] = 0x7F    # a key: the whole row
    got = B.sjd_pool_attention_shared(pool, 0, q, _i32(at), window, group_begin=_begin(groups)).float().cpu().numpy()
    for m, p in enumerate(at):
        if m // window == 1 and p >= 258:
            assert np.isnan(got[m][:heads // kvh]).all() and np.array_equal(got[m][heads // kvh:], clean[m][heads // kvh:])
        else:
            assert np.array_equal(got[m], clean[m])
    assert pool.fault() == 0


@pytest.mark.gpu
def test_exponents_of_any_size():
    groups = [(2, [150, 330, 129])]
    pool, lens = _filled(groups, 1, 1, 64, 20, exps=(-9, -6))
    rng = np.random.default_rng(21)
    q, at = _queries(3 * 8, 2, 64, 22), _window_pos(lens, 8, (8, 8, 1))
    pool.exps[:, :, 1] = torch.from_numpy(rng.integers(-100, 101, tuple(pool.exps[:, :, 1].shape)).astype(np.int8)).cuda()
    _check(pool, q, at, 8, _begin(groups))
    for e in (-100, 5, 127, -128):   # all alike; those beyond +-100 are read as +-100
        pool.exps[:, :, 1] = e
        _check(pool, q, at, 8, _begin(groups))
    # one token takes nearly all of the weight and its values are small: the others' still count
    pool.exps[:, :, 1] = 5
    pool.exps[pool.table[:, 0].long(), :, 1, :, 0] = -30
    _check(pool, _queries(3 * 8, 2, 64, 23, spread=4.0), at, 8, _begin(groups))


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kvh,hd,window", [(2, 1, 64, 8), (8, 1, 128, 40)])
@pytest.mark.parametrize("keys,behind,size,scale", [((-100, -100), None, 2.0 ** -60, 0.0), ((-128, -128), None, 1.3, 1e-20),
                                                   ((-100, 0), None, 1.3, 1e-30), ((-24, -24), None, 1.3, 0.0), ((-8, -5), -128, 2.0 ** -60, 0.0), ((-8, -5), -100, 1.3, 1e-20)])
def test_keys_queries_and_scales_of_any_size(heads, kvh, hd, window, keys, behind, size, scale):
    """A factor of the scores may be as small as it likes, of keys that a row sees and of those that it does not: hidden ones stay hidden.  Rows at -1 hold the
    smallest number that there is.  behind: exponents of the blocks behind a sequence."""
    groups = [(2, [150, 330, 129, 200])]
    pool, lens = _filled(groups, 1, kvh, hd, 48)
    rng = np.random.default_rng(49)
    pool.exps[:, :, 0] = torch.from_numpy(rng.integers(keys[0], keys[1] + 1, tuple(pool.exps[:, :, 0].shape)).astype(np.int8)).cuda()
    if behind is not None:
        for b, n in enumerate(lens):
            if n % 64:
                pool.exps[pool.table[b, n // 64].long(), :, 0, :, -(-n % 64 // 16):] = behind
    q, at = _queries(len(lens) * window, heads, hd, 50, spread=size), _window_pos(lens, window, (window, window, 1, window - 3))
    q[torch.tensor(at) < 0] = torch.tensor(1, dtype=torch.int16).view(torch.bfloat16).cuda()
    _check(pool, q, at, window, _begin(groups), scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kvh,hd,window", [(2, 1, 64, 8), (8, 1, 128, 40)])
@pytest.mark.parametrize("keys", [(-100, 100), (14, 18), (24, 28), (30, 34), (90, 100)])
def test_scores_that_32_bits_hold_without_fractions(heads, kvh, hd, window, keys):
    """Scores of 2^25 and far more, where the key with the largest takes all of the weight (what is next to it is behind by more than scores are off)."""
    groups = [(2, [150, 330, 129, 200])]
    pool, lens = _filled(groups, 1, kvh, hd, 48)
    rng = np.random.default_rng(49)
    pool.exps[:, :, 0] = torch.from_numpy(rng.integers(keys[0], keys[1] + 1, tuple(pool.exps[:, :, 0].shape)).astype(np.int8)).cuda()
    _check(pool, _queries(len(lens) * window, heads, hd, 50), _window_pos(lens, window, (window, window, 1, window - 3)), window, _begin(groups))


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kvh,hd,window", [(2, 1, 64, 8), (8, 1, 128, 40)])
@pytest.mark.parametrize("far", [17, 30, 60])
@pytest.mark.parametrize("pages", [[0, 1], [0], [1, 2], [3, 4], [0, 1, 2, 3, 4, 5]])
def test_scores_far_below_zero_do_not_change_those_of_other_keys(heads, kvh, hd, window, far, pages):
    """Some of the pages hold keys whose scores are -2^27 and far less: tiles of only such, or of such and others; at last all tiles."""
    groups = [(3, [250, 330, 229, 300])]
    pool, lens = _filled(groups, 1, kvh, hd, 51)
    q, at = _queries(len(lens) * window, heads, hd, 52).abs(), _window_pos(lens, window, (window, window, 1, window - 3))
    for page in pages:
        of = pool.table[:, page][pool.table[:, page] >= 0].long()
        raw = pool.pages.view(torch.uint8)[of, :, 0]
        pool.pages.view(torch.uint8)[of, :, 0] = raw & 0x7F | 0x80
        pool.exps[of, :, 0] = far
    pool.pages.view(torch.uint8)[:, :, 0][(pool.pages.view(torch.uint8)[:, :, 0] & 0x7F) == 0x7F] = 0x10   # (behind the sequences)
    _check(pool, q, at, window, _begin(groups))


@pytest.mark.gpu
def test_maxima_that_grow_from_tile_to_tile():
    """Scores that rise by far more than a reference may lag behind, and that fall."""
    groups = [(8, [1300, 1200])]
    pool, lens = _filled(groups, 1, 1, 128, 24, exps=(-8, -8))
    for back in (False, True):
        at = torch.arange(-(-max(lens) // 64))
        step = (at.flip(0) if back else at) // 2 - 10
        for b in range(2):
            live = pool.table[b, :at.numel()] >= 0
            pool.exps[pool.table[b, :at.numel()][live].long(), 0, 0] = step[live.cpu()].clamp(-9, -2)[:, None, None].to(torch.int8).cuda()
        _check(pool, _queries(2 * 6, 4, 128, 25, spread=2.0), _window_pos(lens, 6), 6, _begin(groups))


@pytest.mark.gpu
def test_infinite_and_nan_queries_stay_in_their_row():
    groups = [(2, [200, 300])]
    pool, lens = _filled(groups, 1, 1, 64, 26)
    q, at = _queries(2 * 5, 2, 64, 27), _window_pos(lens, 5)
    want = _check(pool, q, at, 5, None)
    q[3, 1, 7], q[8, 0, 2] = float("nan"), float("inf")
    got = B.sjd_pool_attention_shared(pool, 0, q, _i32(at), 5)
    bad = torch.zeros(10, 2, dtype=torch.bool)
    bad[3, 1] = bad[8, 0] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], want[~bad])


@pytest.mark.gpu
def test_strides_and_unaligned_queries():
    groups = [(2, [180, 300, 210])]
    pool, lens = _filled(groups, 1, 2, 64, 28)
    m, at = 3 * 7, _window_pos(lens, 7)
    whole = torch.randn(m, 4 * 64 + 12, device="cuda").bfloat16()
    out = torch.full((m, 4 * 64 + 20), 3.0, device="cuda").bfloat16()
    for off in (0, 4, 8):
        q = whole[:, off:off + 256].unflatten(1, (4, 64))
        want = _check(pool, q.contiguous(), at, 7, _begin(groups))
        got = B.sjd_pool_attention_shared(pool, 0, q, _i32(at), 7, group_begin=_begin(groups), out=out[:, 4:260].unflatten(1, (4, 64)))
        assert torch.equal(got, want) and (out[:, :4] == 3).all() and (out[:, 260:] == 3).all()


@pytest.mark.gpu
def test_what_is_wrong_on_the_device_is_told():
    groups = [(3, [250, 300])]
    pool, lens = _filled(groups, 1, 1, 64, 29)
    q, at = _queries(2 * 3, 2, 64, 30), _window_pos(lens, 3)
    want = _check(pool, q, at, 3, None)

    def told(pos=at, seqs=None, begin=None):
        out = B.sjd_pool_attention_shared(pool, 0, q, _i32(pos), 3, seqs=_i32(seqs) if seqs else None, group_begin=_i32(begin) if begin else None)
        code = pool.fault()
        pool.clear()
        return code, out

    for begin in ([0, 1], [1, 2], [0, 3], [-1, 2]):
        code, out = told(begin=begin)
        assert code == B.SJD_ERR_BAD_ARG
        assert (out.float() - want.float()).abs().max() < 0.05 * want.float().abs().max()   # (nothing is shared then)
    for pos in (at[:5] + [64 * pool.table.shape[1]], at[:5] + [-2]):
        code, out = told(pos)
        assert code == B.SJD_ERR_BAD_ARG and (out[5] == 0).all()
    code, out = told(seqs=[0, 2])
    assert code == B.SJD_ERR_BAD_ARG and (out[3:] == 0).all()
    assert told(seqs=[-1, 1])[0] == B.SJD_ERR_BAD_ARG
    for b, page in ((1, 4), (0, 1)):   # no page where rows see keys: those keys are left out
        kept = pool.table[b, page].item()
        for gone in (-1, pool.refs.numel(), 1 << 30):
            pool.table[b, page] = gone
            assert told()[0] == B.SJD_ERR_BAD_ARG
        pool.table[b, page] = kept
    assert told()[0] == 0
    three = _filled([(3, [250, 300, 280])], 1, 1, 64, 29)[0]
    B.sjd_pool_attention_shared(three, 0, q[:2], _i32([249, 299]), 1, group_begin=_i32([0, 2]), seqs=_i32([0, 2]))
    assert three.fault() == 0
    for begin in ([0, 2, 1], [0, 4, 3], [2, 1, 3], [0, 1, 2]):
        B.sjd_pool_attention_shared(three, 0, q[:3], _i32([249, 299, 279]), 1, group_begin=_i32(begin))
        assert three.fault() == B.SJD_ERR_BAD_ARG
        three.clear()


@pytest.mark.gpu
def test_in_a_graph_on_another_stream_and_with_a_workspace_of_its_own():
    groups = [(4, [300, 400, 350])]
    pool, lens = _filled(groups, 1, 2, 128, 31)
    q, at, begin = _queries(3 * 8, 4, 128, 32), _i32(_window_pos(lens, 8)), _begin(groups)
    want = B.sjd_pool_attention_shared(pool, 0, q, at, 8, group_begin=begin)
    ws = torch.empty(int(B.lib().sjd_pool_attention_shared_workspace_bytes(pool.ref, 3, 8, 4)), dtype=torch.uint8, device="cuda")
    out, again, graph = torch.zeros_like(want), torch.zeros_like(want), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.sjd_pool_attention_shared(pool, 0, q, at, 8, group_begin=begin, out=out)
        B.sjd_pool_attention_shared(pool, 0, q, at, 8, group_begin=begin, out=again, ws=ws)
    big = _queries(3 * 400, 4, 128, 33)
    B.sjd_pool_attention_shared(pool, 0, big, _i32([i % 300 for i in range(1200)]), 400)   # (a larger workspace: the graph keeps its own)
    stream = torch.cuda.Stream()
    for _ in range(5):
        out.zero_(), again.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        assert torch.equal(out, want) and torch.equal(again, want)
    assert pool.fault() == 0


@pytest.mark.gpu
def test_pages_behind_four_gigabytes():
    groups = [(5, [500, 420, 390]), (2, [200, 300])]
    pool, lens = _filled(groups, 8, 8, 128, 44)
    q, at, begin = _queries(5 * 4, 16, 128, 45), _i32(_window_pos(lens, 4)), _begin(groups)
    n, count = pool.pages.shape[0], 4400   # (a megabyte each)
    pages = torch.zeros((count, *pool.pages.shape[1:]), dtype=torch.uint8, device="cuda")
    exps = torch.zeros((count, *pool.exps.shape[1:]), dtype=torch.int8, device="cuda")
    pages[count - n:], exps[count - n:] = pool.pages.view(torch.uint8).flip(0), pool.exps.flip(0)
    refs = torch.zeros(count, dtype=torch.int32, device="cuda")
    refs[count - n:] = pool.refs.flip(0)
    far = B.CachePool(pages.view(torch.float8_e4m3fn), exps, torch.where(pool.table >= 0, count - 1 - pool.table, pool.table), refs)
    for layer in (0, 7):
        want = B.sjd_pool_attention_shared(pool, layer, q, at, 4, group_begin=begin)
        assert torch.equal(B.sjd_pool_attention_shared(far, layer, q, at, 4, group_begin=begin), want)
    assert pool.fault() == 0 and far.fault() == 0


@pytest.mark.gpu
def test_the_same_as_attention_of_every_sequence():
    """Beside sjd_pool_attention, whose weights have other roundings (2^-8 as well)."""
    groups = [(10, [900, 801, 1200, 700])]
    pool, lens = _filled(groups, 1, 2, 64, 34)
    q, at = _queries(4 * 16, 8, 64, 35), _window_pos(lens, 16)
    a, b = _check(pool, q, at, 16, None), B.sjd_pool_attention(pool, 0, q, _i32(at), 16)
    assert torch.linalg.vector_norm(a.float() - b.float()) <= 2.0 ** -8 * torch.linalg.vector_norm(b.float())


@pytest.mark.gpu
def test_binding_refuses_what_does_not_fit():
    pool, lens = _filled([(2, [150, 160])], 1, 1, 64, 36)
    q, at = _queries(4, 2, 64, 37), _i32(_window_pos(lens, 2))
    for kw in (dict(window=3), dict(group_begin=_i32([0])), dict(group_begin=_begin([(0, [1, 1])]).long()), dict(in_pos=at.cpu()), dict(q=q[:3]), dict(seqs=_i32([0])),
               dict(out=q.float()), dict(ws=torch.zeros(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            B.sjd_pool_attention_shared(pool, 0, **{**dict(q=q, in_pos=at, window=2), **kw})
    with pytest.raises(B.SJDError):
        B.sjd_pool_attention_shared(pool, 0, q.float(), at, 2)
    with pytest.raises(B.SJDError):
        B.sjd_pool_attention_shared(pool, 0, q, at, 2, ws=torch.zeros(256, dtype=torch.uint8, device="cuda"))
