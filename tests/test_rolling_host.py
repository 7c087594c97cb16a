"""Host side of the rolling cache's operators: refusals, rotary tables and scalings, and the oracle itself."""
import ctypes
import math

import numpy as np
import pytest

from oracle import rolling
from paper_2508_16201_b200 import specvlm

BAD, SHAPE, SMALL = specvlm.ERR_INVALID_ARG, specvlm.ERR_UNSUPPORTED_SHAPE, specvlm.ERR_WORKSPACE_TOO_SMALL


def _kv(paged=True):
    kv = specvlm.KvStruct()
    kv.k = kv.v = kv.seq_lens = 0x1000
    kv.n_layers, kv.n_kv_heads, kv.head_dim, kv.n_blocks, kv.max_blocks = 2, 4, 128, 10, 4
    kv.block_tokens, kv.max_seq_len = (64, 256) if paged else (256, 256)
    kv.block_table = 0x2000 if paged else None
    kv.stride_token, kv.stride_head, kv.stride_block, kv.stride_layer = 128, 128 * 64, 128 * 64 * 4, 128 * 64 * 40
    return kv


def _rows():
    return specvlm.RowsStruct(0x3000, 1024, 1024, 1024, 128)


def _rope():
    r = specvlm.RopeStruct()
    r.turns, r.rot_dim, r.n_axes, r.factor = 0x4000, 128, 1, 1.0
    return r


def _append(kv=None, rope=None, q=None, q_out=None, k=None, v=None, batch=1, n_new=1, heads=28, lens=0x5000, no_q=False):
    f = ctypes.byref
    q, q_out = (None, None) if no_q else (q or _rows(), q_out or _rows())
    return specvlm.lib().specvlm_rope_append_kv(f(kv or _kv()), f(rope or _rope()), q and f(q), q_out and f(q_out),
                                                f(k or _rows()), f(v or _rows()), batch, n_new, heads, None, None, lens, 0,
                                                None, None)


def _with(make, **fields):
    x = make()
    for name, value in fields.items():
        setattr(x, name, value)
    return x


def test_rope_append_refusals():
    rope, rows = (lambda **f: _with(_rope, **f)), (lambda **f: _with(_rows, **f))
    assert _append(n_new=0) == BAD and _append(n_new=257) == BAD and _append(lens=None) == BAD and _append(batch=0) == BAD
    assert _append(heads=-1) == BAD and _append(heads=0) == BAD                # rows of queries, but no head
    assert _append(no_q=True) == BAD and _append(q=rows(p=None)) == BAD and _append(q_out=rows(p=None)) == BAD
    assert _append(k=rows(p=None)) == BAD and _append(v=rows(p=None)) == BAD
    assert _append(k=rows(p=0x3008)) == BAD and _append(v=rows(stride_token=1028)) == BAD and _append(q=rows(stride_head=4)) == BAD
    assert _append(rope=rope(turns=None)) == BAD
    for n in (0, 8, 24, 144, -16):
        assert _append(rope=rope(rot_dim=n)) == SHAPE
    for n in (0, 4):
        assert _append(rope=rope(n_axes=n)) == BAD
    assert _append(rope=rope(factor=math.inf)) == BAD and _append(rope=rope(factor=math.nan)) == BAD
    three = rope(n_axes=3)
    for sections in ((16, 24, 23), (-8, 48, 24), (64, 64, 0), (2 ** 31 - 1, 2 ** 31 - 1, 66)):
        for a, x in enumerate(sections):
            three.sections[a] = x
        assert _append(rope=three) == BAD
    assert _append(kv=_with(_kv, head_dim=96)) == SHAPE and _append(kv=_with(_kv, max_seq_len=257)) == BAD


def test_page_refusals():
    L, f = specvlm.lib(), ctypes.byref
    big = 1 << 24
    reserve = lambda kv=None, table=0x2000, ref=0x6000, batch=2, n=3, ws=0x10000, size=big: L.specvlm_reserve_pages(  # noqa: E731
        f(kv or _kv()), table, ref, batch, n, None, ws, size, None, None)
    assert reserve(table=None) == BAD and reserve(ref=None) == BAD and reserve(n=-1) == BAD and reserve(ws=None) == BAD
    assert reserve(ws=0x10001) == BAD and reserve(batch=0) == BAD and reserve(batch=1025) == SHAPE
    assert reserve(size=L.specvlm_pages_workspace_bytes(f(_kv()), 2) - 1) == SMALL
    assert reserve(kv=_with(_kv, block_tokens=96)) == SHAPE and reserve(kv=_with(_kv, max_blocks=3)) == BAD
    release = lambda window=1, sinks=0, table=0x2000: L.specvlm_release_pages(f(_kv()), table, 0x6000, 2, window, sinks, None, None)  # noqa: E731
    assert release(window=0) == BAD and release(sinks=-1) == BAD and release(table=None) == BAD
    fork = lambda kv=None, ref=0x6000, parents=0x7000, n=2, table=0x8000, lens=0x9000: L.specvlm_fork_pages(  # noqa: E731
        f(kv or _kv()), ref, 2, parents, n, table, lens, None, None)
    assert fork(ref=None) == BAD and fork(parents=None) == BAD and fork(table=None) == BAD and fork(lens=None) == BAD
    assert fork(n=0) == BAD and fork(n=1025) == SHAPE and fork(kv=_kv(paged=False)) == BAD
    assert fork(table=0x2000) == BAD and fork(table=0x2000 - 16) == BAD and fork(table=0x2000 + 16) == BAD      # onto the old table
    assert fork(lens=0x1000) == BAD and fork(lens=0x1004) == BAD
    compact = lambda ws=0x10000, size=big, table=0x2000: L.specvlm_compact_pages(f(_kv()), table, 0x6000, 2, None, ws, size, None, None)  # noqa: E731
    assert compact(ws=None) == BAD and compact(size=100) == SMALL and compact(table=None) == BAD
    for batch in (0, -1, 1025):
        assert L.specvlm_pages_workspace_bytes(f(_kv()), batch) == 0
    assert specvlm.status_string(specvlm.ERR_NO_PAGES) == "too few free pages"


def test_turns_are_the_fraction_of_a_turn():
    f = np.array([1.0, 0.25, 1e-7, 0.0, 2 * math.pi, 7.5, -0.5, 5e-324])
    turns = (ctypes.c_uint64 * len(f))()
    assert specvlm.lib().specvlm_rope_turns((ctypes.c_double * len(f))(*f), len(f), turns) == 0
    for x, t in zip(f, turns):
        whole = np.longdouble(x) / (2 * np.arctan2(np.longdouble(0), np.longdouble(-1)))
        want = whole - np.floor(whole)
        off = abs(np.longdouble(t) / np.longdouble(2.0 ** 64) - want)
        assert min(off, 1 - off) <= 2.0 ** -63, (x, t)             # an extended number carries 64 bits
    for bad in (math.inf, math.nan):
        assert specvlm.lib().specvlm_rope_turns((ctypes.c_double * 1)(bad), 1, turns) == BAD
    assert specvlm.lib().specvlm_rope_turns((ctypes.c_double * 1)(1.0), 0, turns) == BAD


@pytest.mark.parametrize("rot", [16, 64, 128])
def test_frequencies_of_the_scalings(rot):
    n, base, scale, ctx, low, high = rot // 2, 10000.0, 8.0, 8192.0, 1.0, 32.0
    plain = rolling.frequencies(rot, base)
    get = lambda s: specvlm.rope_frequencies(rot, base, s, scale, ctx, low, high).numpy()  # noqa: E731
    tight = dict(rtol=1e-14, atol=0)
    np.testing.assert_allclose(get(specvlm.ROPE_PLAIN), plain, **tight)
    np.testing.assert_allclose(get(specvlm.ROPE_LINEAR), plain / scale, **tight)
    stretched = get(specvlm.ROPE_BASE)
    assert stretched[0] == 1.0
    np.testing.assert_allclose(stretched[-1], plain[-1] / scale, rtol=1e-12)       # the longest wave by exactly the scale
    ramp, bands = get(specvlm.ROPE_RAMP), get(specvlm.ROPE_BANDS)
    for i in range(n):
        turns = ctx * plain[i] / (2 * math.pi)
        a = max(math.floor(rot * math.log(ctx / (high * 2 * math.pi)) / (2 * math.log(base))), 0)
        b = min(math.ceil(rot * math.log(ctx / (low * 2 * math.pi)) / (2 * math.log(base))), rot - 1)
        share = min(max((i - a) / (b - a), 0.0), 1.0)
        np.testing.assert_allclose(ramp[i], plain[i] * (1 - share) + plain[i] / scale * share, **tight)
        want = plain[i] if turns > high else plain[i] / scale if turns < low else None
        if want is None:
            t = (turns - low) / (high - low)
            want = plain[i] * t + plain[i] / scale * (1 - t)
        np.testing.assert_allclose(bands[i], want, **tight)


def test_frequencies_refusals():
    for args in ((2,), (17,), (0,), (64, 1.0), (64, math.inf), (64, 1e4, 5), (64, 1e4, specvlm.ROPE_LINEAR, 0.0),
                 (64, 1e4, specvlm.ROPE_BANDS, 8.0, 0.0), (64, 1e4, specvlm.ROPE_RAMP, 8.0, 8192.0, 32.0, 1.0)):
        with pytest.raises(specvlm.SpecvlmError):
            specvlm.rope_frequencies(*args)


def test_oracle_pages_by_hand():
    """Two branches of a sequence of six tokens on pages of four: the begun page is shared until one of them writes."""
    pool, table, lens = rolling.Pool(8, 4), [[-1, -1, -1]], [0]
    assert pool.reserve(table, lens, [6], 12) == ([], True, []) and table == [[0, 1, -1]]
    table, lens = pool.fork(table, [6], [0, 0])
    assert table == [[0, 1, -1]] * 2 and pool.ref[:3] == [2, 2, 0]
    assert pool.reserve(table, lens, [3, 1], 12) == ([(1, 2, 2)], True, [])         # the first copies, the second keeps the page
    assert table == [[0, 2, 3], [0, 1, -1]] and pool.ref == [2, 1, 1, 1, 0, 0, 0, 0]
    assert pool.reserve(table, [9, 7], [4, 0], 12)[2] == [0]                        # no room
    assert pool.reserve(table, [9, 8], [3, 4], 12) == ([], True, []) and table[1] == [0, 1, 4]
    pool.release(table, [9, 8], 3, 1)
    assert table == [[0, 2, 3], [0, 1, -1]] and pool.ref == [2, 1, 1, 1, 0, 0, 0, 0]
    pool.release(table, [9, 8], 1, 1)
    assert table == [[0, -1, 3], [0, 1, -1]] and pool.ref == [2, 1, 0, 1, 0, 0, 0, 0]
    assert pool.compact(table) == ([(3, 2)], 3) and table == [[0, -1, 2], [0, 1, -1]] and pool.ref == [2, 1, 1, 0, 0, 0, 0, 0]
    pool.release(table, [0, 8], 12, 0)
    assert table == [[-1, -1, -1], [0, 1, -1]] and pool.ref == [1, 1, 0, 0, 0, 0, 0, 0]
    assert pool.reserve(table, [0, 8], [12, 4], 12) == ([], True, []) and table == [[2, 3, 4], [0, 1, 5]]
    before = [list(row) for row in table], list(pool.ref)
    assert pool.reserve([[-1, -1, -1]], [0], [12], 12) == ([], False, []) and before == (table, pool.ref)   # two pages are left


def test_oracle_window_is_the_definition():
    assert rolling.window_keys(9, 3, 2) == [0, 1, 7, 8, 9] and rolling.window_keys(2, 3, 2) == [0, 1, 2]
    assert rolling.window_keys(-1, 3, 2) == [] and rolling.window_keys(5, 1, 0) == [5]
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(2, 4, 8)), rng.normal(size=(2, 9, 8)), rng.normal(size=(2, 9, 8))
    out, lse = rolling.attention_window(q, k, v, 9, 1, 0, 0.3)                       # each token sees itself alone
    np.testing.assert_allclose(out[1, 3], v[1, 8])
    np.testing.assert_allclose(lse[0, 0], 0.3 * (q[0, 0] @ k[0, 7]))


def test_window_refusals():
    def call(kv=None, q=0x3000, batch=2, heads=8, n_q=1, window=5, sinks=0, scale=0.1, out=0x4000, ws=0x10000, size=1 << 26):
        return specvlm.lib().specvlm_window_attn(ctypes.byref(kv or _kv()), q, batch, heads, n_q, window, sinks, scale, out, None,
                                                 ws, size, None, None)
    assert call(window=0) == BAD and call(window=-1) == BAD and call(sinks=-1) == BAD and call(n_q=0) == BAD
    assert call(q=None) == BAD and call(out=None) == BAD and call(q=0x3008) == BAD and call(scale=0.0) == BAD and call(scale=math.nan) == BAD
    assert call(heads=0) == BAD and call(heads=9) == BAD and call(batch=0) == BAD
    assert call(n_q=10) == SHAPE and call(heads=4 * 17) == SHAPE
    assert call(kv=_with(_kv, max_seq_len=2 ** 31 - 255, max_blocks=2 ** 25)) == SHAPE
    assert call(heads=4 * 8, n_q=6, batch=128) == SHAPE
    assert call(kv=_with(_kv, n_kv_heads=7300), heads=7300 * 16, n_q=9) == SHAPE   # 144 rows run in groups of 16, as CTAs of a grid
    assert call(heads=4 * 8, n_q=6, ws=None) == BAD and call(heads=4 * 8, n_q=6, ws=0x10010) == BAD
    assert call(heads=4 * 8, n_q=6, size=16) == SMALL
    assert call(kv=_with(_kv, head_dim=96)) == SHAPE and call(kv=_with(_kv, n_kv_heads=0)) == BAD
    size = lambda *a: specvlm.lib().specvlm_window_attn_workspace_bytes(ctypes.byref(_kv()), *a)  # noqa: E731
    assert size(2, 32, 6, 5, 0) > 0 and size(2, 8, 1, 5, 0) > 0
    for bad in ((0, 8, 1, 5, 0), (2, 8, 0, 5, 0), (2, 8, 1, 0, 0), (2, 8, 1, 5, -1), (2, 68, 1, 5, 0), (2, 9, 1, 5, 0), (2, 8, 10, 5, 0)):
        assert size(*bad) == 0, bad


def test_a_window_workspace_is_no_larger_than_the_whole_caches():
    for tokens in (64, 1000, 6400, 50000):
        kv = _with(_kv, max_seq_len=tokens)
        for heads, n_q in ((28, 1), (32, 6), (64, 8)):
            whole = specvlm.lib().specvlm_attn_workspace_bytes(ctypes.byref(kv), 4, heads, n_q - 1)
            for window, sinks in ((1, 0), (512, 64), (4096, 4), (2 ** 31 - 1, 2 ** 31 - 1)):
                assert specvlm.lib().specvlm_window_attn_workspace_bytes(ctypes.byref(kv), 4, heads, n_q, window, sinks) <= whole
