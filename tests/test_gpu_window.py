"""Attention with a window and sinks (specvlm_window_attn) against the plain statement in 64 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import rolling
from paper_2508_16201_b200 import specvlm, synth

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.fixture(autouse=True)
def _built_in_choice():
    yield
    specvlm.debug_set_attn_splits(0)
    specvlm.debug_set_window_kernel(0)


def _cache(L, H, D, lens, n_q, window, sinks, *, page, seed, release=True, extra=0):
    """A cache in which every row that no query of the call sees is NaN, in K and in V, and pages without another row are
    not mapped; and the host's copies [b][L][H][len][D]."""
    B, max_len = len(lens), max(max(lens), 1) + extra
    if page:
        need = [-(-n // page) for n in lens]
        table = synth.page_table(B, -(-max_len // page), sum(need) + 2, need, seed, "cuda")
        shape = (L, sum(need) + 2, H, page, D)
    else:
        table, shape = None, (L, B, H, max_len, D)
    k, v = (synth.randn_bf16(shape, "cuda", seed, t) for t in ("K", "V"))
    seen_k, seen_v = (torch.full(shape, NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    host = []
    for b, n in enumerate(lens):
        keys = set()
        for t in range(n_q):
            keys |= set(rolling.window_keys(n - n_q + t, window, sinks))
        keys = torch.tensor(sorted(keys), dtype=torch.long, device="cuda")
        pos = torch.arange(n, device="cuda")
        if page:
            row = table[b].long()
            where, every = (row[keys // page], keys % page), (row[pos // page], pos % page)
        else:
            where, every = (torch.full_like(keys, b), keys), (torch.full_like(pos, b), pos)
        for x, y in ((seen_k, k), (seen_v, v)):
            x[:, where[0], :, where[1]] = y[:, where[0], :, where[1]]
        host.append([x[:, every[0], :, every[1]].permute(1, 2, 0, 3).double().cpu().numpy() for x in (k, v)])   # [L][H][n][D]
        if page and release:
            held = set((keys // page).tolist())
            for j in range(table.shape[1]):
                if j not in held:
                    table[b, j] = -1
    cache = specvlm.KvCache(seen_k, seen_v, torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len, table)
    return cache, host


def _reference(q, host, lens, window, sinks, scale):
    """out, lse and sum of p |v| per output, by the definition."""
    L, B, n_q, Hq, D = q.shape
    qd = q.double().cpu().numpy()
    out, absum, lse = np.zeros(qd.shape), np.zeros(qd.shape), np.full(qd.shape[:-1], -np.inf)
    for b, n in enumerate(lens):
        k, v = host[b]
        group = Hq // k.shape[1]
        for t in range(n_q):
            keys = rolling.window_keys(n - n_q + t, window, sinks)
            if not keys:
                continue
            kk, vv = k[:, :, keys], v[:, :, keys]
            x = scale * np.einsum("lhgd,lhkd->lhgk", qd[:, b, t].reshape(L, -1, group, D), kk)
            m = x.max(-1, keepdims=True)
            e = np.exp(x - m)
            s = e.sum(-1, keepdims=True)
            out[:, b, t] = np.einsum("lhgk,lhkd->lhgd", e / s, vv).reshape(L, Hq, D)
            absum[:, b, t] = np.einsum("lhgk,lhkd->lhgd", e / s, np.abs(vv)).reshape(L, Hq, D)
            lse[:, b, t] = (m + np.log(s)).reshape(L, Hq)
    return out, absum, lse


def _compare(got, lse, ref):
    """Every probability is rounded to bf16 (2^-8 of it), the output too (2^-8); the logits come from fp32 sums of at most 128
    exact products (128 x 2^-24 of their absolute sum, below 40 here: 3e-4 of a logit at most, which is a factor of the
    probability), the exponentials are good to 2^-21: 2^-11 of the sum of p |v| covers both.  The lse has the logits'
    error, 3e-4, and the logarithm's, 2^-20 of its value."""
    out, absum, want = ref
    tol = 2.0 ** -8 * np.abs(out) * (1 + 2.0 ** -8) + (2.0 ** -8 + 2.0 ** -11) * absum
    g = got.double().cpu().numpy()
    assert np.all(np.isfinite(g))
    assert np.all(np.abs(g - out) <= tol), (np.abs(g - out) / np.maximum(tol, 1e-30)).max()
    x = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(x), np.isneginf(want))
    fine = np.isfinite(want)
    assert np.all(np.abs(x[fine] - want[fine]) <= 3e-4 + 2.0 ** -20 * np.abs(want[fine]))


def _run(L, Hq, H, D, n_q, lens, window, sinks, *, page=0, seed=0, splits=0, release=True, extra=0, kernels=(1, 2, 3)):
    """kernels: with more than 16 rows per KV head the tensor cores, groups of 16 rows and a warp for each, whatever the choice would be."""
    cache, host = _cache(L, H, D, lens, n_q, window, sinks, page=page, seed=seed, release=release, extra=extra)
    q = synth.randn_bf16((L, len(lens), n_q, Hq, D), "cuda", seed, "Q")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    specvlm.debug_set_attn_splits(splits)
    scale = 1.0 / math.sqrt(D)
    ref = _reference(q, host, lens, window, sinks, scale)
    for kernel in kernels if Hq // H * n_q > 16 else (0,):
        specvlm.debug_set_window_kernel(kernel)
        lse = torch.full(q.shape[:-1], 7.0, dtype=torch.float32, device="cuda")
        out = specvlm.window_attn(cache, q, window, sinks, scale, out=torch.full_like(q, NAN), lse=lse, d_status=st)
        assert int(st) == 0
        _compare(out, lse, ref)


# (query heads, KV heads, head_dim, n_q): up to 16 rows a KV head, up to 64, up to 128, 144
FORMS = [(7, 1, 128, 1), (8, 2, 64, 1), (8, 2, 64, 4), (16, 2, 128, 6), (8, 1, 64, 8), (16, 1, 128, 8), (28, 2, 64, 9), (1, 1, 64, 9),
         (16, 1, 128, 9)]
LENS = [1, 9, 64, 65, 130, 331, 640, 1000]


@pytest.mark.parametrize("Hq,H,D,n_q", FORMS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (63, 64), (64, 0), (65, 1), (130, 5), (200, 65), (333, 130),
                                          (64, 1000), (10 ** 6, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows_and_sinks(Hq, H, D, n_q, window, sinks):
    _run(2, Hq, H, D, n_q, LENS, window, sinks, page=64, seed=window % 100)


@pytest.mark.parametrize("Hq,H,D,n_q", FORMS)
@pytest.mark.parametrize("page", [0, 128, 320])
@pytest.mark.parametrize("splits", [0, 1, 3, 40])
def test_caches_and_splits(Hq, H, D, n_q, page, splits):
    """Contiguous caches and pages of several tiles, a CTA per item and slices cut anywhere."""
    _run(1, Hq, H, D, n_q, [700, 3, 129, 1500], 250, 70, page=page, seed=page + splits, splits=splits)


@pytest.mark.parametrize("Hq,H,D", [(7, 1, 128), (4, 1, 64), (16, 1, 128)])
@pytest.mark.parametrize("length", list(range(186, 200)) + [255, 256, 257, 320])
def test_every_alignment_of_a_window(Hq, H, D, length):
    _run(1, Hq, H, D, 3, [length, length + 64], 70, 17, page=64, seed=length)


@pytest.mark.parametrize("n_q,Hq", [(1, 4), (3, 4), (8, 8), (9, 14)])
def test_sequences_shorter_than_the_window_of_queries(n_q, Hq):
    """Queries before the sequence's first token see nothing: zeros, and an lse of -inf; empty sequences among them."""
    _run(2, Hq, 1, 64, n_q, [0, 1, n_q - 1, n_q, 0, 200], 50, 2, page=64, seed=1)
    _run(2, Hq, 1, 128, n_q, [0, 0], 50, 2, page=0, seed=1)


@pytest.mark.parametrize("L,B,Hq,H,D,n_q,window,sinks,page", [
    (1, 1, 28, 4, 128, 1, 1024, 4, 0), (1, 1, 28, 4, 128, 1, 4096, 64, 64), (28, 2, 28, 4, 128, 1, 512, 4, 64),
    (1, 4, 64, 8, 128, 6, 2048, 128, 64), (3, 2, 40, 8, 128, 6, 1000, 33, 0), (2, 30, 8, 2, 64, 1, 333, 0, 64),
    (1, 130, 4, 1, 64, 1, 100, 3, 64)])
def test_larger_calls(L, B, Hq, H, D, n_q, window, sinks, page):
    """Calls that the built-in choice gives to clusters, to slices of the tile list, and to the tensor cores."""
    _run(L, Hq, H, D, n_q, [5000 - 97 * (b % 20) for b in range(B)], window, sinks, page=page, seed=L + B, kernels=(0, 1, 2, 3))


@pytest.mark.parametrize("L,B,H", [(1, 2, 1), (1, 3, 4), (1, 5, 4), (2, 8, 2), (3, 11, 2), (1, 20, 5), (4, 20, 2)])
@pytest.mark.parametrize("Hq,D,n_q", [(4, 128, 6), (4, 64, 9), (16, 128, 8), (13, 64, 7)])
def test_items_of_every_number(L, B, H, Hq, D, n_q):
    """From two items to 160: clusters of eight, four, two and one CTAs, and slices; sequences shorter than a cluster's tiles and
    empty ones among them."""
    lens = [[700, 0, 1, 129, 350, 64, 900][(b * 3 + b // 7) % 7] for b in range(B)]
    _run(L, Hq * H, H, D, n_q, lens, 260, 70, page=64, seed=B)


@pytest.mark.parametrize("Hq,D,n_q", [(7, 128, 1), (4, 64, 2), (8, 128, 4), (16, 128, 9), (9, 64, 9)])
@pytest.mark.parametrize("window,sinks,page", [(1, 0, 64), (16, 33, 0), (50, 4, 128), (62, 64, 64), (121, 0, 0)])
def test_many_items_of_short_windows(Hq, D, n_q, window, sinks, page):
    """280 items of three tiles at most, whose copies leave out the slices that no query sees."""
    lens = [0, 1, 15, 16, 17, 40, 63, 64, 65, 100, 127, 128, 129, 150, 190, 191, 192, 193, 300, 333, 350, 400, 555, 600, 640, 700, 701, 777]
    _run(5, Hq * 2, 2, D, n_q, lens, window, sinks, page=page, seed=window, kernels=(0, 2, 3))


@pytest.mark.parametrize("seed", range(40))
def test_random_windows(seed):
    rng = np.random.default_rng(1000 + seed)
    D = int(rng.choice([64, 128]))
    group, n_q = int(rng.integers(1, 17)), int(rng.choice([1, 1, 1, 2, 5, 7, 9]))
    H, L, B = int(rng.choice([1, 1, 2, 3])), int(rng.integers(1, 5)), int(rng.integers(1, 9))
    top = int(rng.choice([70, 300, 1500]))
    lens = [int(rng.integers(0, top + 1)) for _ in range(B)]
    window, sinks = int(np.exp(rng.uniform(0, 8))), int(rng.choice([0, 0, 1, 4, 63, 64, 65, int(rng.integers(0, 500))]))
    _run(L, group * H, H, D, n_q, lens, window, sinks, page=int(rng.choice([0, 64, 128, 256])), seed=seed, splits=int(rng.choice([0, 0, 1, 5])),
         extra=int(rng.choice([0, 100])))


def test_a_roomy_cache_and_mapped_pages():
    """Room behind the longest sequence; pages out of the window still mapped."""
    _run(2, 8, 1, 128, 1, [100, 400], 90, 5, page=0, seed=2, extra=5000)
    _run(2, 16, 2, 128, 5, [100, 400], 90, 5, page=64, seed=2, extra=5000, release=False)


def test_a_window_of_everything_is_plain_attention():
    lens, L, Hq, H, D = [700, 129], 2, 16, 2, 128
    for n_q in (1, 6):
        cache, _ = _cache(L, H, D, lens, n_q, 10 ** 6, 0, page=64, seed=3)
        q = synth.randn_bf16((L, 2, n_q, Hq, D), "cuda", 3, "Q")
        a = specvlm.window_attn(cache, q, 700, 0, 0.1)
        b = specvlm.verify_attn(cache, q, n_q - 1, 0.1) if n_q > 1 else specvlm.draft_decode_attn(cache, q[:, :, 0].contiguous(), 0.1)[:, :, None]
        assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -6        # two roundings of values below 1 at most, and P's


def test_rising_maxima_across_the_gap():
    """Sinks whose logits are far below, and far above, those of the window: the running maximum moves by hundreds."""
    for factor in (0.01, 30.0):
        for Hq, n_q in ((4, 1), (8, 6), (16, 8)):
            lens, W, S = [1000], 300, 40
            cache, host = _cache(1, 1, 128, lens, n_q, W, S, page=64, seed=4)
            blk = cache.block_table[0, :1].long()
            cache.k[:, blk, :, :S] = (cache.k[:, blk, :, :S].float() * factor).to(torch.bfloat16)
            host[0][0][:, :, :S] = cache.k[:, blk, :, :S][:, 0].double().cpu().numpy()
            q = synth.randn_bf16((1, 1, n_q, Hq, 128), "cuda", 4, "Q")
            lse = torch.empty(q.shape[:-1], dtype=torch.float32, device="cuda")
            ref = _reference(q, host, lens, W, S, 0.1)
            x = np.abs(ref[2]).max()
            for kernel in (1, 2, 3):
                specvlm.debug_set_window_kernel(kernel)
                out = specvlm.window_attn(cache, q, W, S, 0.1, lse=lse)
                # as _compare, the logits' fp32 sums growing with the factor
                tol = 2.0 ** -8 * np.abs(ref[0]) * (1 + 2.0 ** -8) + (2.0 ** -8 + 2.0 ** -11 * max(1.0, factor)) * ref[1]
                assert np.all(np.abs(out.double().cpu().numpy() - ref[0]) <= tol)
                assert np.abs(lse.double().cpu().numpy() - ref[2]).max() <= 3e-4 * max(1.0, factor) + 2.0 ** -20 * x


def test_a_page_that_is_needed_and_not_mapped_is_reported():
    for Hq, n_q in ((4, 1), (8, 6)):
        for bad in (-1, 10 ** 6):
            cache, _ = _cache(1, 1, 128, [500, 100], n_q, 200, 5, page=64, seed=5)
            cache.block_table[0, 6] = bad
            q = synth.randn_bf16((1, 2, n_q, Hq, 128), "cuda", 5, "Q")
            for splits, kernel in ((0, 1), (1, 2), (3, 0), (0, 3)):
                specvlm.debug_set_attn_splits(splits)
                specvlm.debug_set_window_kernel(kernel)
                st = torch.zeros(1, dtype=torch.int32, device="cuda")
                out = specvlm.window_attn(cache, q, 200, 5, 0.1, d_status=st)
                assert int(st) == specvlm.ERR_INVALID_ARG and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("L,B,H,Hq,n_q,splits,W", [
    (1, 2, 2, 8, 1, 0, 700), (1, 20, 4, 16, 1, 0, 700), (1, 20, 4, 16, 1, 3, 700), (4, 20, 4, 16, 1, 1, 700),       # up to 16 rows
    (1, 2, 2, 16, 6, 0, 300), (1, 15, 4, 32, 5, 0, 300),                                        # groups of 16 rows
    (1, 3, 4, 64, 6, 0, 3000), (1, 6, 4, 64, 6, 0, 3000), (1, 15, 4, 64, 6, 0, 3000),           # clusters on the tensor cores
    (4, 20, 4, 24, 4, 0, 64), (4, 20, 4, 40, 9, 0, 1)])                                         # a warp for 16 rows
def test_what_a_cta_that_gives_up_leaves(L, B, H, Hq, n_q, splits, W):
    """Rows that the CTA has a part of keep what was there, the others are whole; the call says so, and the next is not
    disturbed."""
    S, D, group = 70, 128, Hq // H
    lens = [W + 300 - 30 * (b % 10) for b in range(B)]
    cache, host = _cache(L, H, D, lens, n_q, W, S, page=64, seed=8)
    q = synth.randn_bf16((L, B, n_q, Hq, D), "cuda", 8, "Q")
    specvlm.debug_set_attn_splits(splits)
    ws = torch.full((max(256, specvlm.window_attn_workspace_bytes(cache, B, Hq, n_q, W, S)),), 0xFF, dtype=torch.uint8, device="cuda")
    want, want_lse = torch.empty_like(q), torch.empty(q.shape[:-1], dtype=torch.float32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = specvlm.debug_window_give_up(cache, q, W, S, 0.1, want, want_lse, ws, st)
    assert n > 0 and int(st) == 0
    _compare(want, want_lse, _reference(q, host, lens, W, S, 0.1))
    for lost in sorted({0, 1, n // 2, n - 1}):
        out, lse = torch.full_like(q, 7.0), torch.full_like(want_lse, 7.0)
        st.zero_()
        assert specvlm.debug_window_give_up(cache, q, W, S, 0.1, out, lse, ws, st, lost_cta=lost) == n
        kept, left = lse == want_lse, lse == 7.0
        assert bool((kept ^ left).all())
        assert torch.equal(out[kept], want[kept]) and bool((out[left] == 7.0).all())
        # a KV head's rows, 16 of them at least, stand or fall together; one item, on slices the items that the CTA has a part of
        rows = left.view(L, B, n_q, H, group).permute(0, 1, 3, 2, 4).reshape(-1, n_q * group)
        parts = [p for p in rows.split(16, dim=1)]
        assert all(bool((p == p[:, :1]).all()) for p in parts)
        items = int(rows.any(1).sum())
        lost_parts = sum(int(p[:, 0].sum()) for p in parts)
        assert (items == 1 and lost_parts in (1, len(parts))) if splits != 3 else items <= 2
        assert int(st) == (specvlm.ERR_TIMEOUT if items else 0) and (items > 0 or lost == n - 1)


def test_captured_calls_on_growing_sequences_and_one_workspace():
    """Two captured calls (decode and verification) share a workspace; lengths and tables change between the replays."""
    L, Hq, H, D, W, S = 2, 16, 2, 128, 200, 5
    cache, host = _cache(L, H, D, [400, 900], 6, 10 ** 6, 0, page=64, seed=6)
    q = synth.randn_bf16((L, 2, 6, Hq, D), "cuda", 6, "Q")
    q1 = q[:, :, :1].contiguous()
    sizes = [specvlm.window_attn_workspace_bytes(cache, 2, Hq, n, W, S) for n in (1, 6)]
    ws = torch.full((max(sizes),), 0xFF, dtype=torch.uint8, device="cuda")
    calls, graphs = [], []
    for x in (q1, q):
        out, lse = torch.empty_like(x), torch.empty(x.shape[:-1], dtype=torch.float32, device="cuda")
        calls.append((x, out, lse))
        specvlm.window_attn(cache, x, W, S, 0.1, out=out, lse=lse, ws=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            specvlm.window_attn(cache, x, W, S, 0.1, out=out, lse=lse, ws=ws)
        graphs.append(g)
    for lens in ([400, 900], [7, 613], [64, 1], [399, 0]):
        cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x, out, lse in calls:
            short = [[y[:, :, :n] for y in h] for h, n in zip(host, lens)]
            _compare(out, lse, _reference(x, short, lens, W, S, 0.1))


def test_two_streams_at_once():
    lens, W, S = [900, 500], 300, 9
    cache, host = _cache(2, 2, 64, lens, 1, W, S, page=64, seed=7)
    qs = [synth.randn_bf16((2, 2, 1, 8, 64), "cuda", 7, "Q%d" % i) for i in range(4)]
    torch.cuda.synchronize()
    results = []
    for q in qs:
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            lse = torch.empty(q.shape[:-1], dtype=torch.float32, device="cuda")
            results.append((specvlm.window_attn(cache, q, W, S, 0.125, lse=lse), lse))
    torch.cuda.synchronize()
    for q, (out, lse) in zip(qs, results):
        _compare(out, lse, _reference(q, host, lens, W, S, 0.125))


def test_rolling_step():
    """The operators as they are used: reserve, rotate and append, attend, release; branches of it; the pool compacted.  Every
    step's attention equals that of the plain statement over all tokens so far."""
    L, B, Hq, H, D, W, S, page, max_len = 2, 2, 8, 2, 64, 150, 70, 64, 1000
    pool = 24
    k, v = (torch.full((L, pool, H, page, D), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((B, -(-max_len // page)), -1, dtype=torch.int32, device="cuda")
    cache = specvlm.KvCache(k, v, torch.zeros(B, dtype=torch.int32, device="cuda"), max_len, table)
    ref = torch.zeros(pool, dtype=torch.int32, device="cuda")
    freq = rolling.frequencies(D, 1e4)
    rope = specvlm.Rope(torch.from_numpy(freq))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(0)
    keys, values, lens = [np.zeros((L, H, 0, D)) for _ in range(B)], [np.zeros((L, H, 0, D)) for _ in range(B)], [0] * B

    for step in range(40):
        n = int(rng.choice([1, 1, 4, 9])) if step else 9
        q, nk, nv = synth.randn_bf16((L, B, n, Hq + 2 * H, D), "cuda", step, "qkv").split((Hq, H, H), dim=3)
        specvlm.reserve_pages(cache, ref, n, d_status=st)
        turned = specvlm.rope_append_kv(cache, rope, q, nk, nv, d_status=st)
        lse = torch.empty(turned.shape[:-1], dtype=torch.float32, device="cuda")
        out = specvlm.window_attn(cache, turned, W, S, 0.125, lse=lse, d_status=st)
        specvlm.release_pages(cache, ref, window=W, n_sinks=S, d_status=st)
        # the rows as the cache holds them: rotated and rounded (tests of the rotation have its error)
        for b in range(B):
            new = [torch.stack([x[:, int(cache.block_table[b, p // page]), :, p % page] for p in range(lens[b], lens[b] + n)], 2)
                   for x in (cache.k, cache.v)]
            keys[b] = np.concatenate([keys[b], new[0].double().cpu().numpy()], 2)
            values[b] = np.concatenate([values[b], new[1].double().cpu().numpy()], 2)
            lens[b] += n
        assert int(st) == 0 and cache.seq_lens.tolist() == lens
        _compare(out, lse, _reference(turned, list(zip(keys, values)), lens, W, S, 0.125))
        held = sum(int(r) > 0 for r in ref)
        assert held <= B * (W // page + 2 + -(-S // page) + 1)
        if step % 7 == 3:
            specvlm.compact_pages(cache, ref, d_status=st)
            assert int((ref > 0).sum()) == held and bool((ref[:held] > 0).all())
        if step % 10 == 9:                                    # both go on from one of them
            b = int(rng.integers(0, B))
            new_table, new_lens = torch.empty_like(cache.block_table), torch.empty_like(cache.seq_lens)
            specvlm.fork_pages(cache, ref, torch.tensor([b] * B, dtype=torch.int32, device="cuda"), new_table, new_lens, d_status=st)
            cache = specvlm.KvCache(k, v, new_lens, max_len, new_table)
            keys, values, lens = [keys[b]] * B, [values[b]] * B, [lens[b]] * B
