"""The 8-bit paged cache without a GPU: refusals of the entry points, which come before any device is touched, and the oracle's own
pins (e4m3 numbers against torch's, block exponents, page claims by hand)."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from oracle import pool as O
from paper_2410_01699_b200 import binding as B

FAKE = 1 << 20   # an address that no refused call may use


def _pool(**kw):
    f = dict(pages=FAKE, exps=FAKE, table=FAKE, refs=FAKE, status=FAKE, n_pages=8, n_seqs=2, pages_per_seq=4, n_layers=2, n_kv_heads=2,
             head_dim=64)
    f.update(kw)
    return B.sjd_pool(*[f[n] for n, _ in B.sjd_pool._fields_])


BAD_POOLS = [(dict(pages=None), B.SJD_ERR_BAD_ARG), (dict(exps=None), B.SJD_ERR_BAD_ARG), (dict(table=None), B.SJD_ERR_BAD_ARG),
             (dict(status=None), B.SJD_ERR_BAD_ARG), (dict(pages=FAKE + 8), B.SJD_ERR_BAD_ARG), (dict(exps=FAKE + 2), B.SJD_ERR_BAD_ARG),
             (dict(n_pages=0), B.SJD_ERR_BAD_ARG), (dict(n_seqs=0), B.SJD_ERR_BAD_ARG), (dict(pages_per_seq=0), B.SJD_ERR_BAD_ARG),
             (dict(n_layers=0), B.SJD_ERR_BAD_ARG), (dict(n_kv_heads=-1), B.SJD_ERR_BAD_ARG), (dict(head_dim=96), B.SJD_ERR_UNSUPPORTED),
             (dict(pages_per_seq=(1 << 20) + 1), B.SJD_ERR_CAPACITY), (dict(n_seqs=(1 << 17) + 1), B.SJD_ERR_CAPACITY)]


def _append(pool=None, **kw):
    a = dict(layer=0, batch=2, window=4, heads=4, dtype=0, q=FAKE, qs=256, k=FAKE, ks=128, v=FAKE, vs=128, seqs=None, in_pos=FAKE,
             rope=B.make_rope_cfg((32,)), axis=None, out=FAKE, outs=256)
    a.update(kw)
    return B.lib().sjd_pool_append(C.byref(pool or _pool()), a["layer"], a["batch"], a["window"], a["heads"], a["dtype"], a["q"], a["qs"],
                                   a["k"], a["ks"], a["v"], a["vs"], a["seqs"], a["in_pos"],
                                   C.byref(a["rope"]) if a["rope"] is not None else None, a["axis"], a["out"], a["outs"], None)


def _attention(pool=None, **kw):
    a = dict(layer=0, batch=2, window=4, heads=4, dtype=0, q=FAKE, qs=256, seqs=None, in_pos=FAKE, sliding=0, sinks=0, scale=0.0, out=FAKE,
             outs=256, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return B.lib().sjd_pool_attention(C.byref(pool or _pool()), a["layer"], a["batch"], a["window"], a["heads"], a["dtype"], a["q"], a["qs"],
                                      a["seqs"], a["in_pos"], a["sliding"], a["sinks"], a["scale"], a["out"], a["outs"], a["ws"],
                                      a["ws_bytes"], None)


def _manage(pool=None, which="reserve", n=1, p=FAKE, ws=FAKE, ws_bytes=1 << 20):
    pl = C.byref(pool or _pool())
    if which == "reserve":
        return B.lib().sjd_pool_reserve(pl, n, p, p, p, ws, ws_bytes, None)
    if which == "fork":
        return B.lib().sjd_pool_fork(pl, n, p, p, p, None)
    if which == "free":
        return B.lib().sjd_pool_free(pl, n, p, p, None)
    return B.lib().sjd_pool_compact(pl, ws, ws_bytes, None)


@pytest.mark.parametrize("fields,status", BAD_POOLS)
def test_pools_that_do_not_hold_together_are_refused(fields, status):
    p = _pool(**fields)
    assert _append(p) == status
    assert _attention(p) == status
    assert B.lib().sjd_pool_attention_workspace_bytes(C.byref(p), 4, 4) == 0
    assert B.lib().sjd_pool_workspace_bytes(C.byref(p)) == 0
    for which in ("reserve", "fork", "free", "compact"):
        assert _manage(p, which) == status
    assert _manage(_pool(refs=None), "free") == B.SJD_ERR_BAD_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(layer=2), -1), (dict(layer=-1), -1), (dict(batch=0), -1), (dict(window=0), -1), (dict(heads=0), -1), (dict(dtype=2), -3),
    (dict(k=None), -1), (dict(v=None), -1), (dict(in_pos=None), -1), (dict(out=None), -1), (dict(ks=127), -1), (dict(vs=126), -1),
    (dict(ks=129), -1), (dict(qs=255), -1), (dict(qs=254), -1), (dict(outs=257), -1), (dict(k=FAKE + 4), -1), (dict(q=FAKE + 4), -1),
    (dict(dtype=1, v=FAKE + 2), -1), (dict(rope=B.make_rope_cfg((31,))), -1), (dict(rope=B.make_rope_cfg((16, 17))), -1),
    (dict(rope=B.make_rope_cfg((33, -1))), -1), (dict(rope=B.make_rope_cfg((32,), theta=0.0)), -1),
    (dict(rope=B.make_rope_cfg((32,), theta=math.nan)), -1), (dict(rope=B.sjd_rope(0, (C.c_int32 * 3)(32, 0, 0), 0, 0, 1e4)), -1),
    (dict(rope=B.sjd_rope(4, (C.c_int32 * 3)(32, 0, 0), 0, 0, 1e4)), -1), (dict(batch=1 << 20, window=1 << 20), -2)])
def test_append_refuses(kw, status):
    assert _append(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(layer=2), -1), (dict(batch=0), -1), (dict(window=0), -1), (dict(heads=3), -1), (dict(heads=0), -1), (dict(dtype=7), -3),
    (dict(q=None), -1), (dict(in_pos=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(ws=FAKE + 128), -1),
    (dict(qs=252), -1), (dict(qs=258), -1), (dict(outs=258), -1), (dict(q=FAKE + 8), -1), (dict(dtype=1, out=FAKE + 4), -1),
    (dict(sliding=-1), -1), (dict(sinks=-1), -1), (dict(scale=-1.0), -1), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1),
    (dict(ws_bytes=1024), -2), (dict(batch=1 << 20, window=1 << 20), -2), (dict(heads=2 * 32769, qs=2 * 32769 * 64, outs=2 * 32769 * 64), -2)])
def test_attention_refuses(kw, status):
    assert _attention(**kw) == status


def test_page_functions_refuse():
    for which in ("reserve", "fork", "free"):
        assert _manage(which=which, n=-1) == B.SJD_ERR_BAD_ARG
        assert _manage(which=which, p=None) == B.SJD_ERR_BAD_ARG
        assert _manage(which=which, n=B.SJD_POOL_MAX_LIST + 1) == B.SJD_ERR_CAPACITY
        assert _manage(which=which, n=0, p=None) == B.SJD_OK     # nothing to do
    for which in ("reserve", "compact"):
        assert _manage(which=which, ws=None) == B.SJD_ERR_BAD_ARG
        assert _manage(which=which, ws=FAKE + 4) == B.SJD_ERR_BAD_ARG
        assert _manage(which=which, ws_bytes=256) == B.SJD_ERR_CAPACITY


def test_workspaces_are_as_large_as_the_calls_ask_for():
    p = _pool()
    need = B.lib().sjd_pool_attention_workspace_bytes(C.byref(p), 4, 4)
    assert need > 0 and _attention(ws_bytes=need - 1) == B.SJD_ERR_CAPACITY
    need = B.lib().sjd_pool_workspace_bytes(C.byref(p))
    assert need > 0 and _manage(ws_bytes=need - 1) == B.SJD_ERR_CAPACITY


def test_struct_layouts():
    assert C.sizeof(B.sjd_pool) == 5 * 8 + 6 * 4 and C.sizeof(B.sjd_rope) == 6 * 4 + 8


def test_wrapper_refuses_tensors_that_do_not_fit():
    good = dict(pages=torch.zeros(4, 1, 2, 2, 64, 64).to(torch.float8_e4m3fn), exps=torch.zeros(4, 1, 2, 2, 4, dtype=torch.int8),
                table=torch.zeros(2, 3, dtype=torch.int32), refs=torch.zeros(4, dtype=torch.int32))
    pool = B.CachePool(**good)
    for bad in (dict(exps=good["exps"][:, :, :, :, :3]), dict(refs=good["refs"][:3]), dict(table=good["table"].long()),
                dict(pages=good["pages"].float()), dict(table=good["table"].t()), dict(refs=good["refs"][:, None])):
        with pytest.raises(ValueError):
            B.CachePool(**{**good, **bad})
    with pytest.raises(ValueError):
        B.make_rope_cfg(())
    k = torch.zeros(4, 2, 64)
    pos = torch.zeros(4, dtype=torch.int32)
    for kw in (dict(k=k[:3], v=k), dict(k=k, v=k.to(torch.bfloat16)), dict(k=k.transpose(0, 1).contiguous().transpose(0, 1), v=k),
               dict(k=k, v=k, in_pos=pos.long()), dict(k=k, v=k, window=3), dict(k=k, v=k, axis_pos=pos),
               dict(k=k, v=k, q=torch.zeros(4, 4, 32)), dict(k=k, v=k, seqs=pos), dict(k=k, v=k, q=k, q_out=k.to(torch.bfloat16))):
        with pytest.raises(ValueError):
            with torch.device("cpu"):
                B.sjd_pool_append(pool, 0, **{**dict(in_pos=pos, window=2), **kw})
    for window in (0, -2):
        with pytest.raises(ValueError):
            B.sjd_pool_append(pool, 0, k, k, pos, window)
        with pytest.raises(ValueError):
            B.sjd_pool_attention(pool, 0, k, pos, window)
    # one row alone has no stride that matters
    assert B._pool_rows(torch.zeros(3, 131)[:1, :128].view(1, 2, 64), 2, pool, 1, "k") == 128
    with pytest.raises(B.SJDError):
        B.sjd_pool_append(pool, 0, k.half(), k.half(), pos, 2)
    with pytest.raises(B.SJDError):
        B.sjd_pool_attention(pool, 0, k.half(), pos, 2)


# ---------------------------------------------------------------------------------------------------- pins of the oracle
def test_e4m3_numbers_are_torchs():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(np.isnan(every), np.isnan(O.E4M3)) and np.array_equal(every[~np.isnan(every)], O.E4M3[~np.isnan(O.E4M3)])
    rng = np.random.default_rng(0)
    x = np.concatenate((rng.normal(size=4000) * 2.0 ** rng.integers(-12, 9, 4000), (O.E4M3[:126] + O.E4M3[1:127]) / 2, -O.E4M3[:127],
                        [448.0, 464.0, 1e9, -1e9, 2.0 ** -10, 3 * 2.0 ** -10])).astype(np.float32)
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(O.to_e4m3(x), want)
    assert O.to_e4m3([math.nan, math.inf, -math.inf]).tolist() == [0x7F] * 3


def test_block_exponents():
    for top, e in ((448.0, 0), (449.0, 1), (224.0, -1), (224.5, 0), (0.0, 0), (1.0, -8), (1e-45, -100), (3e38, 100)):
        assert O.block_exponent(np.array([0.0, -top, math.nan, math.inf])) == e


def test_claims_by_hand():
    z = lambda *s: np.zeros(s, np.int32)
    pool = O.Pool(np.zeros((8, 1, 2, 1, 64, 64), np.uint8), np.zeros((8, 1, 2, 1, 4), np.int8), z(4, 3) - 1, z(8))
    pool.reserve([0], [0], [100])
    pool.pages[:, ..., 0] = np.arange(8)[:, None, None, None, None]
    assert pool.table[0].tolist() == [0, 1, -1] and pool.refs.tolist() == [1, 1] + [0] * 6
    pool.fork([0, 0], [1, 2], [100, 64])
    assert pool.refs.tolist() == [3, 2] + [0] * 6
    pool.reserve([1, 0], [100, 100], [130, 101])     # page 1: sequence 1 copies it, sequence 0 is its last holder
    assert pool.table.tolist() == [[0, 1, -1], [0, 2, 3], [0, -1, -1], [-1, -1, -1]]
    assert pool.refs.tolist() == [3, 1, 1, 1, 0, 0, 0, 0] and (pool.pages[2, ..., 0] == 1).all()
    pool.free([0, 2], [0, 0])
    assert pool.refs.tolist() == [1, 0, 1, 1, 0, 0, 0, 0]
    pool.compact()
    assert pool.table[1].tolist() == [0, 2, 1] and pool.refs.tolist() == [1, 1, 1] + [0] * 5 and (pool.pages[1, ..., 0] == 3).all()
    for args in (([0, 0], [0, 0], [1, 1]), ([4], [0], [1]), ([0], [0], [193]), ([0, 2], [0, 0], [192, 192])):
        with pytest.raises(O.Refused):
            pool.reserve(*args)


# ------------------------------------------------------------------------------------------------- how attention is shared out
def _equal_ranges(calls):
    """The library's rule (csrc/pool_route.h) for calls (entries, kv_heads, positions, pages_per_seq, window, sliding, sinks, sms)."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "route.cpp"), os.path.join(d, "route")
        with open(src, "w") as f:
            f.write('#include <cstdio>\n#include "pool_route.h"\nint main() {\n  long a[8];\n'
                    '  while (std::scanf("%ld %ld %ld %ld %ld %ld %ld %ld", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7) == 8)\n'
                    '    std::printf("%d\\n", (int)sjd::pool_equal_ranges(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]));\n}\n')
        subprocess.run(["g++", "-std=c++17", "-I" + os.path.join(root, "include"),
                        "-I" + os.path.join(root, "paper_2410_01699_b200", "csrc"), src, "-o", exe], check=True)
        text = "".join(" ".join(str(int(x)) for x in c) + "\n" for c in calls)
        return [bool(int(x)) for x in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()]


def test_places_of_equal_ranges_stay_in_32_bits():
    """Rows of a window at any positions: a unit can have all tiles of its table, a sliding window or not, and 3 more places."""
    rng = np.random.default_rng(3)
    calls = [(512, 8, 4096, 1 << 20, 8, 100, 0, 148), (4096 // 64, 64, 512, 1 << 20, 8, 1, 4, 148)]
    for _ in range(2000):
        entries, kv, window = rng.integers(1, 600), 1 << rng.integers(0, 12), rng.integers(1, 64)
        calls.append((entries, kv, entries * window, 1 << rng.integers(0, 21), window, rng.choice([0, rng.integers(1, 2**31)]), rng.integers(0, 200), 148))
    for c, cut in zip(calls, _equal_ranges(calls)):
        tiles = c[0] * c[1] * (c[3] * 64 // 128 + 3)
        assert not cut or tiles < 1 << 30, c
    # one token of a short and of a long sequence, many of them, more than are looked at
    assert _equal_ranges([(1, 2, 1, 4, 1, 0, 0, 148), (1, 8, 1, 1600, 1, 0, 0, 148), (32, 8, 32, 66, 1, 0, 0, 148), (4, 8, 4, 400, 1, 100, 4, 148),
                          (513, 8, 513, 66, 1, 0, 0, 148)]) == [False, True, True, False, False]
