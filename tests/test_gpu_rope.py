"""Rotary positions and append (specvlm_rope_append_kv) against the plain statement in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

from gpu_util import launches
from oracle import rolling
from paper_2508_16201_b200 import specvlm, synth

pytestmark = pytest.mark.gpu

NAN = float("nan")


def _problem(L, B, n, Hq, H, D, lens, caps, *, page=0, seed=0, packed=True):
    """A cache full of a sentinel (NaN), and the rows of a projection (q, k and v side by side, or each alone)."""
    max_len = max(caps)
    if page:
        need = [-(-c // page) for c in caps]
        table = synth.page_table(B, -(-max_len // page), sum(need) + 2, need, seed, "cuda")
        shape = (L, sum(need) + 2, H, page, D)
    else:
        table, shape = None, (L, B, H, max_len, D)
    k, v = (torch.full(shape, NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = specvlm.KvCache(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len, table)
    if packed:
        rows = synth.randn_bf16((L, B, n, Hq + 2 * H, D), "cuda", seed, "qkv").split((Hq, H, H), dim=3)
    else:
        rows = [synth.randn_bf16((L, B, n, h, D), "cuda", seed, t) for h, t in ((Hq, "q"), (H, "k"), (H, "v"))]
    return cache, rows


def _row(cache, t, b, pos):
    if cache.block_table is None:
        return t[:, b, :, pos]
    page = t.shape[3]
    return t[:, int(cache.block_table[b, pos // page]), :, pos % page]


def _near(got, x, want, factor):
    """Half a step of bf16 (2^-8 of the value) for the rounding; and for a pair (x, y) the sine and cosine, off by less than
    2^-22 each (the angle is cut to 2^-32 of a turn and rounded to fp32: 2^-25 of half a turn, 1e-7 radians; sincospi's own
    error is an ulp, 2^-24), the product with the factor and the three operations of a rotation, 2^-24 each: 2^-20 of the
    largest channel."""
    tol = 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) + 2.0 ** -20 * factor * np.abs(x).max()
    assert np.all(np.abs(got - want) <= tol), np.abs(got - want).max()


def _check(cache, rope_args, rows, q_out, starts, news, positions=None):
    freq, factor, inter, sections = rope_args
    q, k, v = (r.double().cpu().numpy() for r in rows)
    out = q_out.double().cpu().numpy() if q_out is not None else None
    for b, (start, m) in enumerate(zip(starts, news)):
        for t in range(m):
            pos = [start + t] if positions is None else [int(p[b, t]) for p in positions]
            pos = pos * 3 if positions is None and sections else pos
            if out is not None:
                _near(out[:, b, t], q[:, b, t], rolling.rotate(q[:, b, t], pos, freq, factor, inter, sections), factor)
            _near(_row(cache, cache.k, b, start + t).double().cpu().numpy(), k[:, b, t],
                  rolling.rotate(k[:, b, t], pos, freq, factor, inter, sections), factor)
            assert torch.equal(_row(cache, cache.v, b, start + t), rows[2][:, b, t])
    # every other row of the cache still holds the sentinel
    n_rows = sum(news) * cache.k.shape[0] * cache.k.shape[2] * cache.k.shape[4]
    for x in (cache.k, cache.v):
        assert int((~torch.isnan(x)).sum()) == n_rows


SHAPES = [(1, 1, 1, 28, 4, 128), (2, 3, 6, 8, 2, 64), (1, 2, 70, 5, 1, 128), (3, 1, 2, 64, 8, 128), (1, 4, 33, 4, 1, 64),
          (13, 1, 1, 40, 8, 128), (17, 6, 1, 8, 2, 64), (1, 20, 1, 5, 1, 128)]


@pytest.mark.parametrize("L,B,n,Hq,H,D", SHAPES)
@pytest.mark.parametrize("inter,rot,page", [(False, 1.0, 0), (True, 1.0, 64), (False, 0.5, 128), (True, 0.25, 0), (False, 0.75, 64)])
def test_rotation_and_append(L, B, n, Hq, H, D, inter, rot, page):
    rot = max(16, int(rot * D) // 16 * 16)
    lens = [61 + 7 * b for b in range(B)]
    cache, rows = _problem(L, B, n, Hq, H, D, lens, [x + n for x in lens], page=page, seed=n + rot)
    freq = rolling.frequencies(rot, 10000.0)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    rope = specvlm.Rope(torch.from_numpy(freq), interleaved=inter, factor=1.2)
    q_out = specvlm.rope_append_kv(cache, rope, *rows, d_status=st)
    assert int(st) == 0 and cache.seq_lens.tolist() == [x + n for x in lens]
    _check(cache, (freq, 1.2, inter, None), rows, q_out, lens, [n] * B)


@pytest.mark.parametrize("position", [0, 1, 50303, 1000003, 2 ** 31 - 9, -5, -(2 ** 31)])
@pytest.mark.parametrize("inter", [False, True])
def test_far_positions_keep_their_angles(position, inter):
    cache, rows = _problem(1, 1, 8, 4, 2, 64, [0], [8], seed=3)
    freq = specvlm.rope_frequencies(64, 1e6).numpy()
    pos = torch.tensor([[[position + i for i in range(8)]]], dtype=torch.int32, device="cuda")
    q_out = specvlm.rope_append_kv(cache, specvlm.Rope(torch.from_numpy(freq), interleaved=inter), *rows, positions=pos)
    _check(cache, (freq, 1.0, inter, None), rows, q_out, [0], [8], pos.cpu())


@pytest.mark.parametrize("sections", [(16, 24, 24), (64, 0, 0), (0, 0, 64), (1, 62, 1), (40, 24)])
@pytest.mark.parametrize("inter", [False, True])
def test_position_axes(sections, inter):
    L, B, n = 2, 2, 9
    cache, rows = _problem(L, B, n, 28, 4, 128, [3, 70], [12, 79], page=64, seed=4)
    freq = rolling.frequencies(128, 1e6)
    pos = torch.randint(0, 60000, (len(sections), B, n), dtype=torch.int32, generator=torch.Generator().manual_seed(1)).cuda()
    rope = specvlm.Rope(torch.from_numpy(freq), interleaved=inter, sections=sections)
    q_out = specvlm.rope_append_kv(cache, rope, *rows, positions=pos)
    _check(cache, (freq, 1.0, inter, sections), rows, q_out, [3, 70], [n, n], pos.cpu())


@pytest.mark.parametrize("sections", [None, (16, 8, 8)])
@pytest.mark.parametrize("counted", [False, True])
@pytest.mark.parametrize("L,n", [(1, 5), (4, 40)])
def test_padded_batch(sections, counted, L, n):
    """Ragged numbers of new tokens, none and all among them; padding is neither rotated nor appended."""
    news, starts = [n, 0, 1, n - 2], [64, 10, 0, 63]
    lens = [s + m if counted else s for s, m in zip(starts, news)]
    cache, rows = _problem(L, 4, n, 8, 2, 64, lens, [s + m for s, m in zip(starts, news)], page=64, seed=5)
    for r in rows:
        for b, m in enumerate(news):
            r[:, b, m:] = NAN
    rope = specvlm.Rope(torch.from_numpy(rolling.frequencies(64, 1e4)), sections=sections)
    q_out = torch.full_like(rows[0].contiguous(), 7.0)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    specvlm.rope_append_kv(cache, rope, *rows, q_out=q_out, new_lens=torch.tensor(news, dtype=torch.int32, device="cuda"),
                           counted=counted, d_status=st)
    assert int(st) == 0 and cache.seq_lens.tolist() == [s + m for s, m in zip(starts, news)]
    clean = [torch.nan_to_num(r) for r in rows]
    _check(cache, (rolling.frequencies(64, 1e4), 1.0, False, sections), clean, q_out, starts, news)
    for b, m in enumerate(news):
        assert bool((q_out[:, b, m:] == 7.0).all())


def test_in_place_and_strided_and_keys_alone():
    """q_out = q inside the projection's rows, head-major strides, and a call without queries: the same values."""
    L, B, n, Hq, H, D = 2, 2, 3, 8, 2, 128
    rope = specvlm.Rope(torch.from_numpy(rolling.frequencies(96, 1e4)))
    results = []
    for form in ("plain", "in place", "head-major", "keys alone"):
        cache, (q, k, v) = _problem(L, B, n, Hq, H, D, [5, 64], [8, 67], page=64, seed=6)
        out = None
        if form == "head-major":
            q, k, v = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (q, k, v))
            out = torch.empty((B, Hq, n, L, D), dtype=torch.bfloat16, device="cuda").permute(3, 0, 2, 1, 4)
        out = specvlm.rope_append_kv(cache, rope, None if form == "keys alone" else q, k, v, q_out=q if form == "in place" else out)
        results.append((cache.k, cache.v, out if form != "keys alone" else results[0][2]))
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(torch.nan_to_num(a, 9.0), torch.nan_to_num(b, 9.0))
    assert out is None


def test_layer_by_layer_equals_all_layers():
    """The first layer's call counts the tokens, the others find them counted."""
    L, B, n, Hq, H, D = 4, 3, 6, 8, 2, 64
    lens, caps = [1, 64, 100], [7, 70, 106]
    rope = specvlm.Rope(torch.from_numpy(rolling.frequencies(64, 1e4)))
    whole, rows = _problem(L, B, n, Hq, H, D, lens, caps, page=64, seed=7)
    want = specvlm.rope_append_kv(whole, rope, *rows)
    c, _ = _problem(L, B, n, Hq, H, D, lens, caps, page=64, seed=7)
    for layer in range(L):
        one = specvlm.KvCache(c.k[layer:layer + 1], c.v[layer:layer + 1], c.seq_lens, c.max_seq_len, c.block_table)
        got = specvlm.rope_append_kv(one, rope, *(r[layer:layer + 1] for r in rows), counted=layer > 0)
        assert torch.equal(got[0], want[layer])
    assert c.seq_lens.tolist() == caps
    for a, b in ((c.k, whole.k), (c.v, whole.v)):
        assert torch.equal(torch.nan_to_num(a, 9.0), torch.nan_to_num(b, 9.0))


@pytest.mark.parametrize("Hq,H,D,inter,rot", [(4, 1, 64, False, 64), (8, 2, 64, True, 48), (5, 1, 128, False, 32), (0, 3, 64, False, 16)])
@pytest.mark.parametrize("L,B,n", [(7, 2, 3000), (23, 3, 900), (1, 5, 4000)])
def test_many_tokens_of_few_heads(Hq, H, D, inter, rot, L, B, n):
    """Enough tokens for warps that take several layers of one, a number that does not divide the layers among them: the same
    bits as layer by layer, whose calls are smaller; ragged, with a page that is not mapped, and padding left alone."""
    news = [n - 37 * b for b in range(B)]
    starts = [0] + [61 + b for b in range(1, B)]
    caps = [s + n for s in starts]
    freq = torch.from_numpy(rolling.frequencies(rot, 1e4))
    rope = specvlm.Rope(freq, interleaved=inter, factor=1.1)
    results = []
    for whole in (True, False):
        cache, rows = _problem(L, B, n, max(Hq, 1), H, D, starts, caps, page=64, seed=13)
        cache.block_table[B - 1, 2] = -1
        q = rows[0] if Hq else None
        out = torch.full(rows[0].shape, 7.0, dtype=torch.bfloat16, device="cuda") if Hq else None
        new_lens = torch.tensor(news, dtype=torch.int32, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        if whole:
            specvlm.rope_append_kv(cache, rope, q, rows[1], rows[2], q_out=out, new_lens=new_lens, d_status=st)
        else:
            for layer in range(L):
                for b in range(B):                               # one sequence at a time: few tokens a call
                    one = specvlm.KvCache(cache.k[layer:layer + 1], cache.v[layer:layer + 1], cache.seq_lens[b:b + 1].clone(),
                                          cache.max_seq_len, cache.block_table[b:b + 1])
                    cut = [x[layer:layer + 1, b:b + 1] if x is not None else None for x in (q, rows[1], rows[2], out)]
                    specvlm.rope_append_kv(one, rope, *cut[:3], q_out=cut[3], new_lens=new_lens[b:b + 1], d_status=st)
            cache.seq_lens += new_lens
        assert int(st) == specvlm.ERR_INVALID_ARG and cache.seq_lens.tolist() == [s + m for s, m in zip(starts, news)]
        results.append((torch.nan_to_num(cache.k, 9.0), torch.nan_to_num(cache.v, 9.0), out))
    for a, b in zip(*results):
        assert a is None or torch.equal(a, b)
    if Hq:
        for b, m in enumerate(news):
            assert bool((results[0][2][:, b, m:] == 7.0).all()) and not bool((results[0][2][:, b, :m] == 7.0).all(-1).any())


@pytest.mark.parametrize("counted", [False, True])
@pytest.mark.parametrize("n", [2, 60])
def test_sequences_out_of_range_are_left_alone(counted, n):
    """No room, a negative length, a length past the cache, too many or negative new tokens: reported, nothing of them is
    touched; their neighbours are served."""
    news = [n, n, n, n + 1, -1, n, 1]
    starts = [0, 200 - n + 1, -1, 0, 0, 5, 200]
    good = [0, 5]
    lens = [s + m if counted else s for s, m in zip(starts, news)]
    if counted:
        lens[2] = -1
    B = len(news)
    cache, rows = _problem(2, B, n, 4, 1, 64, [0] * B, [200] * B, seed=8)
    cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    rope = specvlm.Rope(torch.from_numpy(rolling.frequencies(64, 1e4)))
    q_out = torch.full((2, B, n, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    specvlm.rope_append_kv(cache, rope, *rows, q_out=q_out, new_lens=torch.tensor(news, dtype=torch.int32, device="cuda"),
                           counted=counted, d_status=st)
    assert int(st) == specvlm.ERR_INVALID_ARG
    assert cache.seq_lens.tolist() == [x + (0 if counted or b not in good else news[b]) for b, x in enumerate(lens)]
    for b in range(B):
        assert bool((q_out[:, b] == 7.0).all()) == (b not in good)
        assert bool(torch.isnan(cache.k[:, b]).all()) == (b not in good)


def test_unmapped_page_is_skipped_and_reported():
    cache, rows = _problem(2, 1, 4, 4, 2, 64, [62], [66], page=64, seed=9)
    second = int(cache.block_table[0, 1])
    for bad in (-1, cache.k.shape[1] + 5):
        cache.block_table[0, 1] = bad
        cache.k.fill_(NAN)
        cache.seq_lens.fill_(62)
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        q_out = specvlm.rope_append_kv(cache, specvlm.Rope(torch.from_numpy(rolling.frequencies(64, 1e4))), *rows, d_status=st)
        assert int(st) == specvlm.ERR_INVALID_ARG
        assert not bool(torch.isnan(q_out).any()) and bool(torch.isnan(cache.k[:, second]).all())
        assert int((~torch.isnan(cache.k)).sum()) == 2 * 2 * 2 * 64                  # two tokens on the first page


def test_captured_call_and_other_stream():
    """A captured append, replayed, keeps counting; and a call on a side stream equals one on the default stream."""
    rope = specvlm.Rope(torch.from_numpy(rolling.frequencies(64, 1e4)))
    for L, n in ((1, 1), (3, 5)):
        cache, rows = _problem(L, 2, n, 8, 2, 64, [0, 30], [6 * n, 30 + 6 * n], seed=10)
        q_out = torch.empty(rows[0].shape, dtype=torch.bfloat16, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            specvlm.rope_append_kv(cache, rope, *rows, q_out=q_out)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            specvlm.rope_append_kv(cache, rope, *rows, q_out=q_out)
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert cache.seq_lens.tolist() == [4 * n, 30 + 4 * n]
        for b, start in enumerate((0, 30)):
            for i, t in itertools.product(range(4), range(n)):
                want = rolling.rotate(rows[1][:, b, t].double().cpu().numpy(), [start + i * n + t], rolling.frequencies(64, 1e4), 1.0, False)
                _near(cache.k[:, b, :, start + i * n + t].double().cpu().numpy(), rows[1][:, b, t].double().cpu().numpy(), want, 1.0)


def test_one_launch_where_the_tokens_are_few_or_counted():
    """In a graph; outside of one the last two calls are a launch too, of a cluster, which a graph would gain nothing by."""
    rope = specvlm.Rope(torch.from_numpy(rolling.frequencies(128, 1e4)))
    for L, B, n, counted, want in ((1, 1, 1, True, 1), (4, 3, 6, True, 1), (1, 1, 1, False, 1), (1, 1, 6, False, 1), (5, 3, 2, False, 2),
                                   (1, 17, 1, False, 2)):
        cache, rows = _problem(L, B, n, 28, 4, 128, [9] * B, [9 + 9 * n] * B, seed=11)
        assert launches(lambda: specvlm.rope_append_kv(cache, rope, *rows, counted=counted)) == want, (L, B, n, counted)


def test_offsets_past_32_bits():
    """A layer whose cache holds more than 2^31 elements: rows behind that land where the strides say."""
    free, _ = torch.cuda.mem_get_info()
    cap, H, D = 2200000, 8, 128
    if free < 12 << 30:
        pytest.skip("needs 12 GB of device memory")
    k = torch.empty((1, 1, H, cap, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    cache = specvlm.KvCache(k, v, torch.tensor([cap - 3], dtype=torch.int32, device="cuda"), cap)
    rows = synth.randn_bf16((1, 1, 3, 16 + 2 * H, D), "cuda", 12, "qkv").split((16, H, H), dim=3)
    freq = rolling.frequencies(128, 1e6)
    k[:, :, :, -4:], v[:, :, :, -4:] = NAN, NAN
    specvlm.rope_append_kv(cache, specvlm.Rope(torch.from_numpy(freq)), *rows)
    assert bool(torch.isnan(k[:, :, :, -4]).all())
    for t in range(3):
        x = rows[1][:, 0, t].double().cpu().numpy()
        _near(k[:, 0, :, cap - 3 + t].double().cpu().numpy(), x, rolling.rotate(x, [cap - 3 + t], freq, 1.0, False), 1.0)
        assert torch.equal(v[:, 0, :, cap - 3 + t], rows[2][:, 0, t])
