"""The 8-bit paged cache on a GPU against oracle/pool.py: pages and counts equal, cached entries bit for bit, attention within bounds that
come from the arithmetic."""
import numpy as np
import pytest
import torch

from oracle import pool as O
from paper_2410_01699_b200 import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy()


def _oracle(pool):
    return O.Pool(_bytes(pool.pages), pool.exps.cpu().numpy(), pool.table.cpu().numpy(), pool.refs.cpu().numpy())


def _same(pool, ref, entries=True):
    assert np.array_equal(pool.table.cpu().numpy(), ref.table)
    assert np.array_equal(pool.refs.cpu().numpy(), ref.refs)
    if entries:
        assert np.array_equal(pool.exps.cpu().numpy(), ref.exps)
        a, b = _bytes(pool.pages), ref.pages
        assert np.array_equal(np.where((a & 0x7F) == 0x7F, 0x7F, a), np.where((b & 0x7F) == 0x7F, 0x7F, b))


def _filled(lens, n_layers, kvh, hd, seed, spare=3, per_seq=None, exps=(-8, -5), n_seqs=None):
    """A pool whose sequence b holds lens[b] positions of normal entries, pages in random order; what lies behind them is anything."""
    rng = np.random.default_rng(seed)
    counts = [-(-n // 64) for n in lens]
    n = sum(counts) + spare
    gen = torch.Generator().manual_seed(seed)
    pages = (torch.randn(n, n_layers, 2, kvh, 64, hd, generator=gen) * 70).clamp(-448, 448).to(torch.float8_e4m3fn)
    table = np.full((n_seqs or len(lens), per_seq or max(max(counts), 1)), -1, np.int32)
    order, at, refs = rng.permutation(n), 0, np.zeros(n, np.int32)
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
        if c and lens[b] % 64:   # rows behind the sequence: any bytes, NaN among them
            tail = pages.view(torch.uint8)[table[b, c - 1], ..., lens[b] % 64:, :]
            tail.copy_(torch.from_numpy(rng.integers(0, 256, tail.shape, dtype=np.uint8)))
            tail[..., ::3] = 0x7F
    refs[order[:at]] = 1
    ex = torch.from_numpy(rng.integers(exps[0], exps[1] + 1, (n, n_layers, 2, kvh, 4)).astype(np.int8))
    return B.CachePool(pages.cuda(), ex.cuda(), torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda())


# ------------------------------------------------------------------------------------------------------------ attention
def _bound(dtype, want):
    """Most that an output may be off.  A weight's planes leave 2^-8 (bf16: two) or 2^-16 (fp32: four) of it, half a step of e4m3 being
    2^-4 of a number; its conversion to fp16 before leaves 2^-11 (bf16; with fp32 the planes hold that rest too).  The largest weight of a
    row in a tile of 128 keys is 2^8 and the smallest step of e4m3 2^-9 (fp32: under the factor 2^-8 of the third and fourth plane): half of
    it is 2^-18 resp. 2^-26 of that weight.  A query's planes leave 2^-16 of an entry (fp32; bf16: nothing) and the same floors of the row's
    largest; a score has about 20 fp32 additions (2^-24 of their magnitudes each) and counts twice, in the numerator and in the sum.  Sums
    over the keys: a tile's products and two roundings a tile, up to 800 tiles of a sequence and the merges, 2^-15.  The output's own
    rounding: half a step."""
    out, mass, floor, reach, flat = want
    two = dtype == "bf16"
    low = 2.0 ** -18 if two else 2.0 ** -26
    score = flat * low + reach * (2.0 ** -19 if two else 2.0 ** -16 + 2.0 ** -19)
    weight = 2.0 ** -8 + 2.0 ** -11 if two else 2.0 ** -16
    return 1.02 * ((weight + 2 * score[..., None] + 2.0 ** -15) * mass + floor * low) + (2.0 ** -8 if two else 2.0 ** -24) * np.abs(out) + 1e-35


def _check_attention(pool, q, in_pos, window, dtype, sliding=0, sinks=0, scale=0.0, seqs=None, layer=0, out=None, ref=None):
    batch = len(in_pos) // window
    seen = _i32(seqs) if seqs is not None else None
    out = B.sjd_pool_attention(pool, layer, q, _i32(in_pos), window, sliding=sliding, sinks=sinks, scale=scale, seqs=seen, out=out)
    exact = (ref or _oracle(pool)).attention(layer, q.float().cpu().numpy(), seqs if seqs is not None else range(batch), in_pos, window,
                                             sliding, sinks, scale)
    want = exact[0]
    got = out.float().cpu().numpy().astype(np.float64)
    assert pool.fault() == 0
    err, tol = np.abs(got - want), _bound(dtype, exact)
    assert np.isfinite(got).all()
    assert (err <= tol).all(), "worst %.3g of its bound at %s" % ((err / tol).max(), np.unravel_index((err / tol).argmax(), err.shape))
    for m, p in enumerate(in_pos):
        if p < 0:
            assert (got[m] == 0).all()
    norm = np.linalg.norm(want)
    if norm > 0:   # (a plane less would leave about 2^-5 resp. 2^-16 of the weights, and 2^-4 resp. 2^-12 of every query's entries)
        assert np.linalg.norm(got - want) / norm <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -18)
    return out


def _window_pos(lens, window, active=None):
    """Positions of windows that end sequences; the first active[b] rows of a window are in use."""
    out = []
    for b, n in enumerate(lens):
        k = window if active is None else active[b]
        out += [n - k + i for i in range(k)] + [-1] * (window - k)
    return out


def _queries(m, heads, hd, dtype, seed, spread=1.3):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(m, heads, hd, generator=g) * spread).to(DT[dtype]).cuda()



@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kvh,hd", [(4, 2, 64), (4, 1, 128), (6, 2, 128), (16, 1, 64), (3, 3, 128)])
@pytest.mark.parametrize("lens", [(1,), (31, 32, 33), (63, 64, 65, 127), (700, 1, 130)])
def test_single_tokens(dtype, heads, kvh, hd, lens):
    pool = _filled(lens, 1, kvh, hd, 5)
    _check_attention(pool, _queries(len(lens), heads, hd, dtype, 1), _window_pos(lens, 1), 1, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,heads,kvh,hd", [(16, 2, 2, 64), (17, 1, 1, 128), (32, 2, 2, 128), (33, 2, 2, 64), (64, 1, 1, 128),
                                                 (65, 1, 1, 64), (16, 8, 2, 64), (43, 3, 1, 128), (64, 4, 1, 64), (5, 7, 1, 128), (200, 2, 1, 64)])
def test_windows(dtype, window, heads, kvh, hd):
    lens = (window, window + 77, 515)
    pool = _filled(lens, 1, kvh, hd, 6)
    _check_attention(pool, _queries(3 * window, heads, hd, dtype, 2), _window_pos(lens, window), window, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sliding,sinks", [(1, 0), (1, 1), (5, 4), (32, 32), (33, 0), (64, 40), (100, 4), (100, 1000), (5000, 4), (2**31 - 1, 2**31 - 1)])
def test_sliding_window_and_sinks(dtype, sliding, sinks):
    lens = (20, 340, 801)
    pool = _filled(lens, 1, 2, 64, 7)
    _check_attention(pool, _queries(3 * 20, 4, 64, dtype, 3), _window_pos(lens, 20), 20, dtype, sliding, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_and_sequences_that_see_nothing(dtype):
    lens, window = (0, 90, 0, 7, 300), 9
    pool = _filled(lens, 1, 1, 128, 8, per_seq=6)
    out = torch.full((5 * window, 2, 128), 7.0, device="cuda").to(DT[dtype])
    _check_attention(pool, _queries(5 * window, 2, 128, dtype, 4), _window_pos(lens, window, (0, 4, 0, 7, 9)), window, dtype, out=out)
    # nothing at all
    out = B.sjd_pool_attention(pool, 0, _queries(4, 2, 128, dtype, 4), _i32([-1] * 4), 1)
    assert (out == 0).all() and pool.fault() == 0


def test_rows_of_a_window_in_any_order():
    lens = (400,)
    pool = _filled(lens, 1, 2, 64, 9)
    pos = [399, 3, -1, 250, 3, 64, 63, 0, 128, 32, 31, 399]
    for sliding, sinks in ((0, 0), (40, 3)):
        _check_attention(pool, _queries(12, 4, 64, "f32", 5), pos, 12, "f32", sliding, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,heads,kvh,hd,n", [(1, 4, 1, 128, 20000), (3, 8, 2, 64, 9999), (32, 2, 2, 128, 4009), (64, 4, 1, 128, 3001)])
def test_long_sequences_are_spread_over_the_device(dtype, window, heads, kvh, hd, n):
    lens = (n, n // 3, n // 40)
    pool = _filled(lens, 1, kvh, hd, 10)
    q = _queries(3 * window, heads, hd, dtype, 6)
    a = _check_attention(pool, q, _window_pos(lens, window), window, dtype)
    for _ in range(3):   # the workspace is ready again, and the order of arrival changes nothing
        assert torch.equal(a, B.sjd_pool_attention(pool, 0, q, _i32(_window_pos(lens, window)), window))


def test_more_positions_than_ranges_are_cut_for():
    window, n = 5000, 5000
    pool = _filled((n, n), 1, 1, 64, 11)
    q = _queries(2 * window, 1, 64, "bf16", 7)
    out = B.sjd_pool_attention(pool, 0, q, _i32(_window_pos((n, n), window)), window)
    assert pool.fault() == 0
    ref = _oracle(pool)
    rows = [0, 1, 31, 127, 128, 2500, 4999, 5000, 7777, 9999]
    for m in rows:   # row by row: a window of one
        want = ref.attention(0, q[m:m + 1].float().cpu().numpy(), [m // window], [m % window], 1)
        assert (np.abs(out[m].float().cpu().numpy() - want[0][0]) <= _bound("bf16", want)[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kvh,hd,sliding,sinks", [(2, 1, 128, 0, 0), (4, 2, 64, 0, 0), (4, 1, 128, 70, 3), (1, 1, 64, 300, 0)])
def test_more_sequences_than_ranges_are_cut_for(dtype, heads, kvh, hd, sliding, sinks):
    """513 sequences and more: a block of threads per unit, one of them with a long sequence."""
    lens = [1 + 37 * i % 210 for i in range(519)] + [9000, 64]
    pool = _filled(lens, 1, kvh, hd, 41)
    _check_attention(pool, _queries(len(lens), heads, hd, dtype, 42), _window_pos(lens, 1), 1, dtype, sliding, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kvh,hd,sliding,sinks", [(2, 1, 128, 0, 0), (2, 2, 64, 100, 5)])
def test_windows_of_more_positions_than_ranges_are_cut_for(dtype, heads, kvh, hd, sliding, sinks):
    """8400 positions: windows of 60 rows, short and empty ones among them, and rows at any positions."""
    window, lens = 60, [60 + 29 * i % 200 for i in range(139)] + [1500]
    pool = _filled(lens, 1, kvh, hd, 43)
    pos = _window_pos(lens, window, [window - 7 * i % 61 for i in range(139)] + [window])
    rng = np.random.default_rng(44)
    pos[-window:] = rng.integers(-1, lens[-1], window).tolist()
    _check_attention(pool, _queries(len(lens) * window, heads, hd, dtype, 45), pos, window, dtype, sliding, sinks)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_nan_of_one_entry_stays_with_the_rows_and_the_entry_that_see_it(dtype, hd):
    """Every head of a row that does not see a NaN is as without it, bit for bit; of the others only the entry."""
    n, window = 100, 20
    pool = _filled((n,), 1, 1, hd, 13)
    q, pos = _queries(window, 2, hd, dtype, 9), _window_pos((n,), window)
    clean = B.sjd_pool_attention(pool, 0, q, _i32(pos), window)
    pool.pages.view(torch.uint8)[int(pool.table[0, 90 // 64]), 0, 1, 0, 90 % 64, 5] = 0xFF
    got = B.sjd_pool_attention(pool, 0, q, _i32(pos), window)
    assert pool.fault() == 0
    for m in range(window):
        bad = torch.isnan(got[m])
        if pos[m] < 90:
            assert torch.equal(got[m], clean[m])
        else:
            assert bad[:, 5].all() and int(bad.sum()) == 2 and torch.equal(got[m][~bad], clean[m][~bad])


def _check_weights(dtype, got, exact, q, ref, in_pos, window, sliding, sinks):
    """Entries against a bound in which no row counts that a query does not see, nor an exponent that such a row has set: keys are weighed
    together with blocks of at most 2^5 times smaller exponents, so that half of the smallest step of a weight (_bound: 2^-18 resp. 2^-26 of
    the largest weight times 2^e) is at most 2^-13 resp. 2^-21 of the row's largest weight on every visible |v_j|.  And the norm of every
    head's output as in _check_attention."""
    out, mass, _, reach, flat = exact
    heads, kvh = q.shape[1], ref.pages.shape[3]
    x, floor = q.float().cpu().numpy().astype(np.float64), np.zeros_like(out)
    for m, at in enumerate(in_pos):
        j = np.arange(at + 1)
        seen = (sliding == 0) | (j > at - sliding) | (j < sinks)
        for h in range(heads):
            (k, ke), (v, ve) = (ref.entries(0, m // window, i, h * kvh // heads, at + 1) for i in range(2))
            s = (k * ke)[seen] @ x[m, h] * x.shape[-1] ** -0.5
            floor[m, h] = np.exp(s.max()) / np.exp(s).sum() * np.abs(v * ve)[seen].sum(0)
    bound = _bound(dtype, (out, mass, np.zeros_like(out), reach, flat)) + 1.02 * 2.0 ** (-13 if dtype == "bf16" else -21) * floor
    assert (np.abs(got - out) <= bound).all(), "worst %.3g of its bound" % (np.abs(got - out) / bound).max()
    norms = np.linalg.norm(got - out, axis=-1) / np.linalg.norm(out, axis=-1)
    assert norms.max() <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -18), "%s: %.3g" % (np.unravel_index(norms.argmax(), norms.shape), norms.max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("factor", [2.0 ** 8, 2.0 ** 12, 2.0 ** 16])
@pytest.mark.parametrize("window,heads,kvh,hd,sliding,sinks", [(4, 2, 2, 128, 0, 0), (12, 4, 2, 64, 0, 0), (24, 1, 1, 128, 0, 0), (40, 2, 1, 64, 0, 0),
                                                             (1, 4, 2, 128, 100, 0), (4, 2, 1, 64, 90, 4), (33, 2, 1, 128, 120, 16)])
def test_a_large_value_that_is_not_seen_takes_nothing_from_the_others(dtype, factor, window, heads, kvh, hd, sliding, sinks):
    """Values of a window's last row, or of a row before a sliding window, that are up to 2^16 times the others' set the exponent of their
    block, while the block's other rows are ordinary ones that a query sees beside those of the blocks around it."""
    lens = (window + sliding + 75, window + 300)
    pool = _filled(lens, 1, kvh, hd, 61)
    pos = _window_pos(lens, window)
    for b, n in enumerate(lens):
        v = torch.randn(n, kvh, hd, generator=torch.Generator().manual_seed(62 + b))
        # full: the window's last row, which its others do not see; sliding: the last row that no row of the window sees
        v[n - window - sliding if sliding else n - 1] *= factor
        B.sjd_pool_append(pool, 0, _rows(n, kvh, hd, "f32", 64 + b) * 0.01, v.cuda(), _i32(list(range(n))), n, seqs=_i32([b]))
    q = _queries(2 * window, heads, hd, dtype, 66)
    got = B.sjd_pool_attention(pool, 0, q, _i32(pos), window, sliding=sliding, sinks=sinks).float().cpu().numpy().astype(np.float64)
    assert pool.fault() == 0
    ref = _oracle(pool)
    exact = ref.attention(0, q.float().cpu().numpy(), (0, 1), pos, window, sliding, sinks)
    if not sliding:   # (without the rows that see the large value)
        rows = [m for m in range(2 * window) if m % window != window - 1]
        exact, got, q, pos, window = tuple(x[rows] for x in exact), got[rows], q[torch.tensor(rows)], [pos[m] for m in rows], window - 1
    _check_weights(dtype, got, exact, q, ref, pos, window, sliding, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_exponents_of_any_size(dtype):
    """Values' exponents from end to end of their range within one sequence; keys' so that no score leaves fp32."""
    lens = (150, 330)
    pool = _filled(lens, 1, 1, 64, 12, exps=(-9, -6))
    rng = np.random.default_rng(1)
    pool.exps[:, :, 1] = torch.from_numpy(rng.integers(-100, 101, tuple(pool.exps[:, :, 1].shape)).astype(np.int8)).cuda()
    _check_attention(pool, _queries(2 * 8, 2, 64, dtype, 8), _window_pos(lens, 8), 8, dtype)
    pool.exps[:, :, 1] = -100                     # all alike, at the lower end
    _check_attention(pool, _queries(2 * 8, 2, 64, dtype, 8), _window_pos(lens, 8), 8, dtype)
    pool.exps[:, :, 1] = 127                      # read as 100
    ref = _oracle(pool)
    _check_attention(pool, _queries(2 * 8, 2, 64, dtype, 8), _window_pos(lens, 8), 8, dtype, ref=ref)
    # one token takes nearly all of the weight and its values are small: the others' still count
    pool.exps[:, :, 1] = 5
    pool.exps[pool.table[:, 0].long(), :, 1, :, 0] = -30
    _check_attention(pool, _queries(2 * 8, 2, 64, dtype, 8, spread=4.0), _window_pos(lens, 8), 8, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,heads,kvh,hd,sliding,sinks", [(1, 4, 1, 128, 0, 0), (3, 8, 2, 64, 0, 0), (20, 2, 2, 128, 0, 0), (40, 2, 1, 64, 700, 70)])
def test_tiles_in_several_parts(dtype, window, heads, kvh, hd, sliding, sinks):
    """Exponents of values far apart in every tile, units that several blocks of threads share, the same again from a graph, and values that are
    NaN where only some rows see them."""
    lens = (5000, 1301, window)
    pool = _filled(lens, 1, kvh, hd, 71, per_seq=80)
    rng = np.random.default_rng(72)
    pool.exps[:, :, 1] = torch.from_numpy(rng.integers(-15, 16, tuple(pool.exps[:, :, 1].shape)).astype(np.int8)).cuda()
    pos, q = _window_pos(lens, window), _queries(3 * window, heads, hd, dtype, 73)
    out = _check_attention(pool, q, pos, window, dtype, sliding, sinks)
    at, again, g = _i32(pos), torch.empty_like(out), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sjd_pool_attention(pool, 0, q, at, window, sliding=sliding, sinks=sinks, out=again)
    for _ in range(3):
        again.zero_()
        g.replay()
        assert torch.equal(again, out)
    raw, table = pool.pages.view(torch.uint8), pool.table.cpu().numpy()
    for b, n in enumerate(lens):
        for key in [n - 1, n - window // 2 - 1] + ([n - sliding, n - sliding - window + 1, sinks - 1] if sliding and n > sliding + window else []):
            raw[table[b, key // 64], 0, 1, rng.integers(kvh), key % 64, rng.integers(hd)] = int(rng.choice([0x7F, 0xFF]))
    got = B.sjd_pool_attention(pool, 0, q, at, window, sliding=sliding, sinks=sinks).float().cpu().numpy()
    exact = _oracle(pool).attention(0, q.float().cpu().numpy(), range(3), pos, window, sliding, sinks)
    assert pool.fault() == 0 and np.isnan(exact[0]).any() and np.array_equal(np.isnan(got), np.isnan(exact[0]))
    fine = ~np.isnan(exact[0])
    assert (np.abs(got - exact[0]) <= _bound(dtype, exact))[fine].all()


def test_a_nan_shows_where_it_is_seen_and_nowhere_else():
    n, window = 100, 20
    for dtype in ("bf16", "f32"):
        for hd in (64, 128):
            pool = _filled((n,), 1, 1, hd, 13)
            q = _queries(window, 2, hd, dtype, 9)
            pos = _window_pos((n,), window)
            clean = B.sjd_pool_attention(pool, 0, q, _i32(pos), window)
            page, row = int(pool.table[0, 90 // 64]), 90 % 64
            pool.pages.view(torch.uint8)[page, 0, 1, 0, row, 5] = 0xFF       # a value of key 90: one entry
            got = B.sjd_pool_attention(pool, 0, q, _i32(pos), window)
            for m in range(window):
                bad = torch.isnan(got[m])
                assert bad[:, 5].all() == (pos[m] >= 90) and not bad[:, :5].any() and not bad[:, 6:].any()
            keep = [i for i in range(hd) if i != 5]
            assert torch.equal(got[:, :, keep], clean[:, :, keep])
            pool.pages.view(torch.uint8)[page, 0, 0, 0, row, 3] = 0x7F       # and of the key itself: the whole row
            got = B.sjd_pool_attention(pool, 0, q, _i32(pos), window)
            for m in range(window):
                assert torch.isnan(got[m]).all() == (pos[m] >= 90) and (pos[m] >= 90 or torch.equal(got[m], clean[m]))
            assert pool.fault() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,heads", [(2, 2), (12, 4), (24, 8)])
def test_nans_at_both_ends_of_sliding_windows(dtype, window, heads):
    """Values that are NaN wherever only some rows see them, in the tiles of many sequences and heads, one after another."""
    lens, sliding, sinks = [300 + 37 * i for i in range(40)], 190, 70
    pool = _filled(lens, 1, 2, 128, 51)
    rng, raw, table = np.random.default_rng(52), pool.pages.view(torch.uint8), pool.table.cpu().numpy()
    for b, n in enumerate(lens):
        for key in [n - 1, n - window, n - sliding, n - sliding - window + 1, sinks - 1, sinks, n // 2]:
            raw[table[b, key // 64], 0, 1, rng.integers(2), key % 64, rng.integers(128)] = int(rng.choice([0x7F, 0xFF]))
    pos = _window_pos(lens, window)
    q = _queries(len(lens) * window, heads, 128, dtype, 53)
    got = B.sjd_pool_attention(pool, 0, q, _i32(pos), window, sliding=sliding, sinks=sinks).float().cpu().numpy()
    exact = _oracle(pool).attention(0, q.float().cpu().numpy(), range(len(lens)), pos, window, sliding, sinks, 0.0)
    assert pool.fault() == 0 and np.isnan(exact[0]).any() and not np.isnan(exact[0]).all()
    assert np.array_equal(np.isnan(got), np.isnan(exact[0]))
    fine = ~np.isnan(exact[0])
    assert (np.abs(got - exact[0]) <= _bound(dtype, exact))[fine].all()


def test_queries_that_are_not_finite_or_zero():
    pool = _filled((80,), 1, 1, 64, 14)
    q = _queries(4, 2, 64, "f32", 10)
    q[0] = 0.0
    q[1, 0, 3] = float("nan")
    q[2, 1, 7] = float("inf")
    q[3] *= 1e-30
    out = B.sjd_pool_attention(pool, 0, q, _i32([79, 79, 79, 79]), 4)
    want = _oracle(pool).attention(0, q.cpu().numpy(), [0], [79] * 4, 4)[0]
    assert torch.isnan(out[1, 0]).all() and torch.isnan(out[2, 1]).all()
    for m, h in ((0, 0), (0, 1), (1, 1), (2, 0), (3, 0), (3, 1)):
        assert np.abs(out[m, h].cpu().numpy() - want[m, h]).max() <= 1e-4 * np.abs(want[m, h]).max()


def test_layers_strides_sequences_and_scale():
    """A layer in the middle of a pool, queries inside a wider matrix, table rows picked by the call (one twice)."""
    lens = (70, 200, 129, 5)
    pool = _filled(lens, 3, 2, 128, 15)
    wide = _queries(4 * 3, 10, 128, "f32", 11)
    q = wide[:, 2:6]
    out = torch.full((12, 7, 128), 3.0, device="cuda")
    seqs = (2, 1, 0, 1)
    pos = _window_pos([lens[s] for s in seqs], 3)
    _check_attention(pool, q, pos, 3, "f32", seqs=seqs, layer=1, scale=0.03, out=out[:, 1:5])
    assert (out[:, 0] == 3).all() and (out[:, 5:] == 3).all()


def test_pages_behind_four_gigabytes():
    """Byte offsets of pages pass 32 bits (a page of 32 layers, 32 heads of 128 is 16.8 MB)."""
    n = 300
    pool = B.CachePool.empty(n, 1, 4, 32, 32, 128)
    ids = [n - 1, 0, 256, 255]
    pool.table[0] = _i32(ids)
    pool.refs[torch.tensor(ids, device="cuda")] = 1
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = torch.randn(250, 32, 128, generator=g, device="cuda"), torch.randn(250, 32, 128, generator=g, device="cuda")
    pos = torch.arange(250, dtype=torch.int32, device="cuda")
    B.sjd_pool_append(pool, 31, k, v, pos, 250)
    q = torch.randn(2, 32, 128, generator=g, device="cuda")
    out = B.sjd_pool_attention(pool, 31, q, _i32([100, 249]), 2)
    assert pool.fault() == 0
    small = B.CachePool.empty(4, 1, 4, 1, 32, 128)       # the same in a pool of one layer
    small.table[0] = _i32([0, 1, 2, 3])
    B.sjd_pool_append(small, 0, k, v, pos, 250)
    assert torch.equal(out, B.sjd_pool_attention(small, 0, q, _i32([100, 249]), 2))
    for i, page in enumerate(ids):
        assert torch.equal(pool.pages[page, 31].view(torch.uint8), small.pages[i, 0].view(torch.uint8))
    used = torch.zeros(n, dtype=torch.bool)
    used[ids] = True
    total = pool.pages.view(torch.uint8).view(n, -1)
    for page in (1, 44, 127, 128, 254, 257, 298):
        assert not total[page].any()


def test_faults_are_reported_and_left_out():
    lens = (100, 100)
    for what, pos, seqs, table in (("position", [100, 64 * 2, 99, -2], None, None), ("sequence", [99, 98, 99, 98], (0, 2), None),
                                   ("page", [99, 98, 99, 98], None, (1, 0, -1)), ("page index", [99, 98, 99, 98], None, (0, 1, 1 << 29))):
        pool = _filled(lens, 1, 1, 64, 16, per_seq=2)
        if table is not None:
            pool.table[table[0], table[1]] = table[2]
        q = _queries(4, 2, 64, "f32", 12)
        out = B.sjd_pool_attention(pool, 0, q, _i32(pos), 2, seqs=_i32(seqs) if seqs else None)
        assert pool.fault() == B.SJD_ERR_BAD_ARG, what
        pool.clear()
        if what == "position":
            assert (out[1] == 0).all() and (out[3] == 0).all() and (out[2] != 0).any()
        elif what == "sequence":
            assert (out[2:] == 0).all() and (out[:2] != 0).any()
        elif table == (1, 0, -1):      # the keys of the page are left out
            ref = _oracle(pool)
            k, v = ref.pages[ref.table[1, 1]][0, 0, 0], ref.pages[ref.table[1, 1]][0, 1, 0]
            e = O.clamp_exp(ref.exps[ref.table[1, 1], 0, :, 0]).repeat(16, -1)[..., None]
            k, v = (O.E4M3[k] * 2.0 ** e[0])[:36], (O.E4M3[v] * 2.0 ** e[1])[:36]
            s = k @ q[2, 0].cpu().numpy().astype(np.float64) / 8
            p = np.exp(s - s.max())
            assert np.abs(out[2, 0].cpu().numpy() - p @ v / p.sum()).max() <= 1e-4 * np.abs(v).max()
        # (position 100 sees a row behind the sequence, where NaN stand: they show)
        assert torch.isfinite(out[torch.tensor(pos) != 100]).all() and (pos[0] != 100 or torch.isnan(out[0]).any())


def test_calls_of_two_streams_and_graphs():
    lens = (3000, 2500)
    pool = _filled(lens, 1, 2, 64, 17)
    q = _queries(2 * 4, 4, 64, "bf16", 13)
    pos = _i32(_window_pos(lens, 4))
    want = B.sjd_pool_attention(pool, 0, q, pos, 4)
    torch.cuda.synchronize()
    ws = [torch.empty_like(pool.attention_ws()) for _ in range(2)]
    outs = [torch.empty_like(q) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    graphs = []
    for s, w, o in zip(streams, ws, outs):
        with torch.cuda.stream(s):
            B.sjd_pool_attention(pool, 0, q, pos, 4, out=o, ws=w)
    torch.cuda.synchronize()
    for s, w, o in zip(streams, ws, outs):
        assert torch.equal(o, want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.sjd_pool_attention(pool, 0, q, pos, 4, out=o, ws=w)
        graphs.append(g)
    q.mul_(0.5)
    want = B.sjd_pool_attention(pool, 0, q, pos, 4)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


# --------------------------------------------------------------------------------------------------------------- append
def _rows(m, heads, hd, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, heads, hd, generator=g) * torch.exp2(torch.randint(-6, 7, (m, heads, 1), generator=g).float())
    return x.to(DT[dtype]).cuda()


def _check_append(pool, layer, q, k, v, in_pos, window, pairs, axis_pos=None, theta=10000.0, interleaved=False, per_axis=False, seqs=None, far=False):
    ref = _oracle(pool)
    hd = k.shape[-1]
    rope = B.make_rope_cfg(pairs, theta, interleaved, per_axis) if pairs else None
    q_out = torch.full_like(q, 9.0, memory_format=torch.contiguous_format)
    B.sjd_pool_append(pool, layer, k, v, _i32(in_pos), window, q=q, q_out=q_out, rope=rope,
                      axis_pos=_i32(axis_pos) if axis_pos is not None else None, seqs=_i32(seqs) if seqs is not None else None)
    kk, qq = k.float().cpu().numpy(), q.float().cpu().numpy()
    if pairs:
        at = np.asarray(axis_pos if axis_pos is not None else [[p] * len(pairs) for p in in_pos])
        angles = O.rope_angles(at, hd, pairs, theta, interleaved, per_axis)
        kk, qq = O.rotate(kk, angles), O.rotate(qq, angles)
    vv = v.float().cpu().numpy()
    for b in range(len(in_pos) // window):
        pos = in_pos[b * window:(b + 1) * window]
        n = sum(p >= 0 for p in pos)
        if n:
            m = slice(b * window, b * window + n)
            ref.append(layer, seqs[b] if seqs is not None else b, pos[0], kk[m], vv[m])
    assert pool.fault() == 0
    _same(pool, ref)
    want = torch.from_numpy(qq).to(q.dtype)
    for m, p in enumerate(in_pos):
        if far and p >= 0:
            # Positions of up to 2^20: the fp64 products of two ways to an angle differ by a few 2^-53 of 2^20 radians, 2^-31.  Where a cosine
            # lies as near as that to a border of fp32 numbers, the two round it to neighbours, 2^-24 apart at most; so do both factors of
            # a pair (a, b): 2^-24 (|a| + |b|), and the three roundings that follow may fall differently by as much again.
            x = q[m].float().cpu()
            pair = (x[:, :hd // 2].abs() + x[:, hd // 2:].abs()).repeat(1, 2)
            assert ((q_out[m].cpu() - want[m]).abs() <= 2.0 ** -23 * pair).all()
        else:
            assert torch.equal(q_out[m].cpu(), want[m] if p >= 0 else torch.full_like(want[m], 9.0))
    return ref


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kvh,hd", [(4, 2, 64), (2, 2, 128), (5, 1, 128)])
@pytest.mark.parametrize("window,lens", [(1, (0, 5, 15, 16, 63, 64)), (7, (0, 9, 10, 60)), (16, (0, 1, 48)), (33, (3, 64)), (150, (17,))])
def test_append_matches_the_definition_bit_for_bit(dtype, heads, kvh, hd, window, lens):
    pool = _filled(lens, 1, kvh, hd, 20, spare=0)
    per_seq = -(-(max(lens) + window) // 64)
    full = _filled([n + window for n in lens], 1, kvh, hd, 21, per_seq=per_seq)
    m = len(lens) * window
    in_pos = [n + i for n in lens for i in range(window)]
    _check_append(full, 0, _rows(m, heads, hd, dtype, 1), _rows(m, kvh, hd, dtype, 2), _rows(m, kvh, hd, dtype, 3), in_pos, window, (hd // 2,))
    del pool


@pytest.mark.parametrize("interleaved,per_axis", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("pairs", [(8, 12, 12), (16, 16), (0, 32), (30, 1, 1), (32,)])
def test_rotary_axes(interleaved, per_axis, pairs):
    pool = _filled((60, 60), 1, 2, 64, 22)
    rng = np.random.default_rng(4)
    axis_pos = rng.integers(-50, 1 << 20, (40, len(pairs))).tolist()
    in_pos = [11 + i for i in range(20)] + [30 + i for i in range(20)]
    _check_append(pool, 0, _rows(40, 4, 64, "f32", 4), _rows(40, 2, 64, "f32", 5), _rows(40, 2, 64, "f32", 6), in_pos, 20, pairs, axis_pos,
                  500.0, interleaved, per_axis, far=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_parts_of_one_matrix_ragged_layers_and_rollback(dtype):
    """q, k and v are slices of the projection's output; some windows are short or empty; a window is written over after a rollback."""
    pool = _filled((90, 200, 64, 130), 2, 2, 128, 23, n_seqs=6)
    qkv = _rows(3 * 10, 8, 128, dtype, 7)
    seqs = (3, 0, 1)
    for starts, active in (((100, 40, 150), (10, 3, 0)), ((103, 41, 150), (5, 10, 10)), ((96, 43, 155), (1, 1, 1))):
        pos = [p + i if i < n else -1 for p, n in zip(starts, active) for i in range(10)]
        _check_append(pool, 1, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], pos, 10, (64,), seqs=seqs)
        qkv = qkv.flip(0)
    # in place, and without queries or rotation
    q = qkv[:, :4].contiguous()
    want = B.sjd_pool_append(pool, 1, qkv[:, 4:6], qkv[:, 6:], _i32(pos), 10, q=q, rope=B.make_rope_cfg((64,)), seqs=_i32(seqs))
    assert B.sjd_pool_append(pool, 1, qkv[:, 4:6], qkv[:, 6:], _i32(pos), 10, q=q, q_out=q, rope=B.make_rope_cfg((64,)), seqs=_i32(seqs)) is q
    live = torch.tensor(pos) >= 0
    assert torch.equal(q[live], want[live])
    ref = _oracle(pool)
    B.sjd_pool_append(pool, 0, qkv[:, 4:6], qkv[:, 6:], _i32(pos), 10, seqs=_i32(seqs))
    for b, s in enumerate(seqs):
        ref.append(0, s, pos[b * 10], qkv[b * 10:b * 10 + 1, 4:6].float().cpu().numpy(), qkv[b * 10:b * 10 + 1, 6:].float().cpu().numpy())
    _same(pool, ref)


def test_append_special_entries():
    pool = _filled((64, 64), 1, 1, 64, 24)
    k, v = _rows(8, 1, 64, "f32", 8), _rows(8, 1, 64, "f32", 9)
    k[0, 0, 3], k[1, 0, 3], v[2, 0, 1], v[3, 0, 2] = float("nan"), float("inf"), -float("inf"), float("nan")
    k[4:], v[4:] = 0.0, 1e-42          # a block of zeros and one of the smallest numbers
    v[5, 0, 0] = 3e38
    in_pos = [16, 17, 18, 19, 32, 33, 34, 35]
    _check_append(pool, 0, _rows(8, 1, 64, "f32", 10), k, v, in_pos, 4, None)


def test_append_reports_faults_and_leaves_them_out():
    for pos, seqs in (([60, 61, 62, 64], None), ([60, -1, 62, -1], None), ([-1, 3, 4, 5], None), ([-5, -1, -1, -1], None),
                      ([126, 127, 128, 129], None), ([1 << 30, (1 << 30) + 1, -1, -1], None), ([0, 1, 2, 3], (7,)), ([0, 1, 2, 3], (-1,)),
                      ([2**31 - 1, -1, -1, -1], None)):
        pool = _filled((70, 70), 1, 1, 64, 25)
        before = pool.pages.view(torch.uint8).clone()
        k = _rows(4, 1, 64, "f32", 11)
        B.sjd_pool_append(pool, 0, k, k, _i32(pos), 4, seqs=_i32(seqs) if seqs else None)
        assert pool.fault() == B.SJD_ERR_BAD_ARG, pos
        if pos[0] != 126:   # (there the first two positions exist: their block is written)
            assert torch.equal(before, pool.pages.view(torch.uint8)) or pos == [60, 61, 62, 64]
    pool = _filled((70, 70), 1, 1, 64, 25)
    pool.table[0, 0], pool.table[1, 0] = -1, 1 << 29
    k = _rows(4, 1, 64, "f32", 11)
    before = pool.pages.view(torch.uint8).clone()
    B.sjd_pool_append(pool, 0, k, k, _i32([5, 6, 5, 6]), 2)
    assert pool.fault() == B.SJD_ERR_BAD_ARG and torch.equal(before, pool.pages.view(torch.uint8))
    pool.clear()
    B.sjd_pool_append(pool, 0, k, k, _i32([66, 67, 66, 67]), 2, seqs=_i32([1, 1]))     # a sequence twice
    assert pool.fault() == B.SJD_ERR_BAD_ARG and torch.equal(before, pool.pages.view(torch.uint8))


# ---------------------------------------------------------------------------------------------------------------- pages
def _random_pool(seed, n=400, n_seqs=40, per_seq=12, layers=2, kvh=1, hd=64):
    g = torch.Generator().manual_seed(seed)
    pool = B.CachePool.empty(n, n_seqs, per_seq, layers, kvh, hd)
    pool.pages.view(torch.uint8).copy_(torch.randint(0, 256, pool.pages.shape, generator=g, dtype=torch.uint8))
    pool.exps.copy_(torch.randint(-128, 128, pool.exps.shape, generator=g, dtype=torch.int8))
    return pool


@pytest.mark.parametrize("seed", range(6))
def test_pages_follow_the_definition_through_a_random_life(seed):
    rng = np.random.default_rng(seed)
    pool = _random_pool(seed, n=(60, 400, 5000)[seed % 3], n_seqs=40, kvh=(1, 3)[seed % 2])
    ref = _oracle(pool)
    lens = np.zeros(40, int)
    refused = 0
    for step in range(40):
        what = rng.choice(["reserve", "reserve", "fork", "free", "compact"])
        n = int(rng.integers(1, 15))
        seqs = rng.permutation(40)[:n].tolist()
        if what == "reserve":
            begin = [int(rng.integers(0, lens[s] + 1)) for s in seqs]
            end = [int(min(12 * 64, b + rng.integers(0, 200))) for b in begin]
            args, call = (seqs, begin, end), (B.sjd_pool_reserve, ref.reserve)
        elif what == "fork":
            empty = [s for s in range(40) if (ref.table[s] == -1).all()][:n]
            src = [int(rng.choice([s for s in range(40) if s not in empty] or [0])) for _ in empty]
            args, call = (src, empty, [int(rng.integers(0, lens[s] + 1)) for s in src]), (B.sjd_pool_fork, ref.fork)
        elif what == "free":
            args, call = (seqs, [int(rng.choice([0, rng.integers(0, lens[s] + 1)])) for s in seqs]), (B.sjd_pool_free, ref.free)
        else:
            args, call = (), (B.sjd_pool_compact, ref.compact)
        call[0](pool, *[_i32(a) for a in args])
        try:
            call[1](*args)
            assert pool.fault() == 0
        except O.Refused:
            refused += 1
            assert pool.fault() in (B.SJD_ERR_CAPACITY, B.SJD_ERR_BAD_ARG)
            pool.clear()
        _same(pool, ref, entries=step % 8 == 7)
        for s in range(40):   # positions without a hole
            have = ref.table[s] >= 0
            lens[s] = 64 * (int(np.argmin(have)) if not have.all() else 12)
    assert refused or seed % 3


def test_every_holder_of_a_page_writes():
    """Fork to many, then all write: the last claim keeps the page, the others copy; and a claim of the parent's earlier pages."""
    pool = _random_pool(9)
    ref = _oracle(pool)
    for f, r, args in ((B.sjd_pool_reserve, ref.reserve, ([7], [0], [300])),
                       (B.sjd_pool_fork, ref.fork, ([7] * 20, list(range(10, 30)), [300] * 10 + [256] * 5 + [1] * 5)),
                       (B.sjd_pool_reserve, ref.reserve, ([7] + list(range(10, 20)), [300] * 11, [310] * 11)),
                       (B.sjd_pool_reserve, ref.reserve, (list(range(20, 30)), [256] * 5 + [0] * 5, [257] * 5 + [64] * 5)),
                       (B.sjd_pool_reserve, ref.reserve, ([12, 7], [0, 70], [300, 80]))):
        f(pool, *[_i32(a) for a in args])
        r(*args)
        assert pool.fault() == 0
        _same(pool, ref)


def test_a_long_list_in_a_large_pool():
    pool = B.CachePool.empty(70000, 3000, 40, 1, 1, 64)
    ref = _oracle(pool)
    rng = np.random.default_rng(2)
    for lo in (0, 1024, 1500):
        seqs = list(range(lo, lo + 1024))
        begin = rng.integers(0, 600, 1024).tolist()
        args = (seqs, begin, [b + int(x) for b, x in zip(begin, rng.integers(0, 1500, 1024))])
        args = (args[0], args[1], [min(e, 2560) for e in args[2]])
        B.sjd_pool_reserve(pool, *[_i32(a) for a in args])
        ref.reserve(*args)
        assert pool.fault() == 0
        _same(pool, ref, entries=False)
    B.sjd_pool_free(pool, _i32(list(range(300, 1300))), _i32([128] * 1000))
    ref.free(list(range(300, 1300)), [128] * 1000)
    _same(pool, ref, entries=False)
    B.sjd_pool_compact(pool)
    ref.compact()
    _same(pool, ref, entries=False)
    empty = list(range(2540, 2990))          # (never reserved; sources are others)
    length = rng.integers(0, 129, len(empty)).tolist()
    src = [300 + i % 700 for i in range(len(empty))]
    length = [n if (ref.table[s, :-(-n // 64)] >= 0).all() else 0 for s, n in zip(src, length)]
    assert len(empty) * 40 > 16384 and sum(length) > 0       # (a block for every child)
    B.sjd_pool_fork(pool, _i32(src), _i32(empty), _i32(length))
    ref.fork(src, empty, length)
    assert pool.fault() == 0
    _same(pool, ref, entries=False)
    taken = next(i for i, n in enumerate(length) if n > 0)
    B.sjd_pool_fork(pool, _i32(src), _i32(empty[:taken] + [empty[taken]] + empty[taken + 1:]), _i32(length))     # one is not empty
    assert pool.fault() == B.SJD_ERR_BAD_ARG
    _same(pool, ref, entries=False)


@pytest.mark.parametrize("call,args", [
    (B.sjd_pool_reserve, ([0, 0], [0, 0], [1, 1])), (B.sjd_pool_reserve, ([40], [0], [1])), (B.sjd_pool_reserve, ([-1], [0], [1])),
    (B.sjd_pool_reserve, ([3], [0], [12 * 64 + 1])), (B.sjd_pool_reserve, ([3], [-1], [5])), (B.sjd_pool_reserve, ([3], [2**31 - 64], [2**31 - 1])),
    (B.sjd_pool_fork, ([0, 0], [5, 5], [10, 10])), (B.sjd_pool_fork, ([0], [1], [10])), (B.sjd_pool_fork, ([0], [0], [10])),
    (B.sjd_pool_fork, ([0, 5], [5, 6], [10, 10])), (B.sjd_pool_fork, ([0], [5], [129])), (B.sjd_pool_fork, ([0], [5], [-1])),
    (B.sjd_pool_fork, ([40], [5], [1])), (B.sjd_pool_fork, ([0], [40], [1])), (B.sjd_pool_fork, ([0], [5], [2**31 - 1])),
    (B.sjd_pool_free, ([0, 1, 0], [0, 0, 0])), (B.sjd_pool_free, ([41], [0])), (B.sjd_pool_free, ([0], [-1]))])
def test_refused_page_calls_change_nothing(call, args):
    pool = _random_pool(11)
    B.sjd_pool_reserve(pool, _i32([0, 1]), _i32([0, 0]), _i32([100, 50]))
    before = _oracle(pool)
    call(pool, *[_i32(a) for a in args])
    assert pool.fault() == B.SJD_ERR_BAD_ARG
    _same(pool, before)
    # a pool with a fault stays as it is until it is cleared
    B.sjd_pool_free(pool, _i32([0]), _i32([0]))
    B.sjd_pool_compact(pool)
    B.sjd_pool_reserve(pool, _i32([2]), _i32([0]), _i32([10]))
    B.sjd_pool_fork(pool, _i32([0]), _i32([5]), _i32([10]))
    _same(pool, before)
    pool.clear()
    B.sjd_pool_fork(pool, _i32([0]), _i32([5]), _i32([10]))
    assert pool.fault() == 0 and pool.table[5, 0] == pool.table[0, 0]


def test_too_few_pages():
    pool = _random_pool(12, n=10)
    B.sjd_pool_reserve(pool, _i32([0, 1]), _i32([0, 0]), _i32([256, 200]))
    before = _oracle(pool)
    B.sjd_pool_reserve(pool, _i32([2, 3]), _i32([0, 0]), _i32([64, 65]))
    assert pool.fault() == B.SJD_ERR_CAPACITY
    _same(pool, before)
    pool.clear()
    B.sjd_pool_reserve(pool, _i32([2, 3]), _i32([0, 0]), _i32([64, 64]))
    assert pool.fault() == 0 and (pool.refs == 1).all()


# ------------------------------------------------------------------------------------------------------ all of it together
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_images_of_one_prompt(dtype):
    """A prompt, three images of it, windows with rolled-back drafts, a captured step, an image that leaves, the rest compacted: after
    every step the attention of each layer is that of the oracle's pool, which went through the same."""
    layers, heads, kvh, hd, window, prompt = 2, 4, 2, 64, 12, 75
    pool = B.CachePool.empty(16, 4, 4, layers, kvh, hd)
    pool.pages.view(torch.uint8).fill_(0x7F)
    ref = _oracle(pool)
    rope = B.make_rope_cfg((8, 12, 12))
    axes = lambda p: (p // 100, p // 9 % 11, p % 9)
    rng = np.random.default_rng(5)
    seed = [100]

    def step(seqs, starts, rows, run=None):
        pos = [s + i if i < n else -1 for s, n in zip(starts, rows) for i in range(max(rows))]
        w = max(rows)
        m = len(pos)
        at = [axes(max(p, 0)) for p in pos]
        for layer in range(layers):
            seed[0] += 1
            qkv = _rows(m, heads + 2 * kvh, hd, dtype, seed[0]) * 0.3
            q, k, v = qkv[:, :heads], qkv[:, heads:heads + kvh], qkv[:, heads + kvh:]
            t = dict(pos=_i32(pos), at=_i32(at), seqs=_i32(seqs))
            call = lambda: B.sjd_pool_attention(pool, layer, B.sjd_pool_append(pool, layer, k, v, t["pos"], w, q=q, rope=rope, axis_pos=t["at"],
                                                                               seqs=t["seqs"]), t["pos"], w, sliding=50, sinks=3, seqs=t["seqs"])
            if run is not None:     # captured once it has run, and replayed
                call()
                torch.cuda.synchronize()
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    out = call()
                g.replay()
            else:
                out = call()
            angles = O.rope_angles(np.asarray(at), hd, (8, 12, 12))
            kk, qq = O.rotate(k.float().cpu().numpy(), angles), torch.from_numpy(O.rotate(q.float().cpu().numpy(), angles)).to(DT[dtype]).float().numpy()
            vv = v.float().cpu().numpy()
            for _ in range(2 if run is not None else 1):
                for b, s in enumerate(seqs):
                    if rows[b]:
                        ref.append(layer, s, starts[b], kk[b * w:b * w + rows[b]], vv[b * w:b * w + rows[b]])
            _same(pool, ref)
            want = ref.attention(layer, qq, seqs, pos, w, 50, 3)
            got = out.float().cpu().numpy()
            live = np.asarray(pos) >= 0
            assert pool.fault() == 0
            assert (np.abs(got - want[0])[live] <= _bound(dtype, want)[live]).all() and (got[~live] == 0).all()

    def both(f, r, *args):
        f(pool, *[_i32(a) for a in args])
        r(*args)
        assert pool.fault() == 0
        _same(pool, ref)

    both(B.sjd_pool_reserve, ref.reserve, [0], [0], [prompt])
    step([0], [0], [prompt])
    both(B.sjd_pool_fork, ref.fork, [0, 0], [1, 2], [prompt, prompt])
    n = [prompt] * 3
    for i in range(4):
        both(B.sjd_pool_reserve, ref.reserve, [0, 1, 2], n, [x + window for x in n])
        step([0, 1, 2], n, [window, window - 3, window], run=i == 2 or None)
        n = [x + int(a) for x, a in zip(n, rng.integers(1, window - 3, 3))]      # so many drafts are accepted
    both(B.sjd_pool_free, ref.free, [0, 2], [0, n[2]])
    both(B.sjd_pool_compact, ref.compact)
    step([2, 1], [n[2], n[1]], [1, 1])
