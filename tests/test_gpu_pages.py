"""Pages of a paged cache (reserve, release, fork, compact) against the plain statement, and a long random run of all of them
with the rows of every sequence followed through it."""
import numpy as np
import pytest
import torch

from gpu_util import launches
from oracle import rolling
from paper_2508_16201_b200 import specvlm, synth

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class State:
    """A pool on the device beside its plain statement."""

    def __init__(self, pool, page, batch, max_len, *, L=2, H=2, D=64, seed=0, unaligned=False):
        self.max_len = max_len
        self.k, self.v = (synth.randn_bf16((L, pool, H, page, D), "cuda", seed, t) for t in ("K", "V"))
        self.plain = rolling.Pool(pool, page)
        self.table = [[-1] * -(-max_len // page) for _ in range(batch)]
        self.lens = [0] * batch
        counts = torch.zeros(pool + 1, dtype=torch.int32, device="cuda")
        self.ref = counts[1:] if unaligned else counts[:pool]         # counts that start off a 16-byte boundary
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self._cache()

    def _cache(self):
        self.cache = specvlm.KvCache(self.k, self.v, _i32(self.lens), self.max_len, _i32(self.table))

    def copies(self, moves):
        """The moves that the plain statement asks for, made on host copies: what the pool has to hold afterwards."""
        k, v = self.k.cpu(), self.v.cpu()
        for src, dst, rows in moves:
            for x in (k, v):
                x[:, dst, :, :rows] = x[:, src, :, :rows].clone()
        return k, v

    def check(self, pool=None, status=0):
        torch.cuda.synchronize()
        assert int(self.status) == status
        self.status.zero_()
        assert self.ref.tolist() == self.plain.ref
        assert self.cache.block_table.tolist() == self.table
        assert self.cache.seq_lens.tolist() == self.lens
        if pool is not None:
            assert torch.equal(self.k.cpu(), pool[0]) and torch.equal(self.v.cpu(), pool[1])

    def reserve(self, new, as_list=True, expect=None):
        specvlm.reserve_pages(self.cache, self.ref, 0 if as_list else new[0], new_lens=_i32(new) if as_list else None, d_status=self.status)
        copies, ok, refused = self.plain.reserve(self.table, self.lens, new, self.max_len)
        status = 0 if ok and not refused else specvlm.ERR_INVALID_ARG if ok else specvlm.ERR_NO_PAGES
        if ok or not refused:                                         # (two reports at once: either may stand)
            if expect is not None:
                assert status == expect
            self.check(self.copies(copies), status)
        return ok

    def set_lens(self, lens):
        self.lens = list(lens)
        self.cache.seq_lens.copy_(_i32(self.lens))

    def release(self, window=None, sinks=0):
        specvlm.release_pages(self.cache, self.ref, window=window, n_sinks=sinks, d_status=self.status)
        self.plain.release(self.table, self.lens, window or 1 << 40, sinks)
        self.check()

    def fork(self, parents):
        table = torch.full((len(parents), len(self.table[0])), 77, dtype=torch.int32, device="cuda")
        lens = torch.full((len(parents),), 77, dtype=torch.int32, device="cuda")
        old = self.cache.block_table.clone()
        specvlm.fork_pages(self.cache, self.ref, _i32(parents), table, lens, d_status=self.status)
        assert torch.equal(old, self.cache.block_table)
        self.table, self.lens = self.plain.fork(self.table, self.lens, parents)
        self.cache = specvlm.KvCache(self.k, self.v, lens, self.max_len, table)
        self.check()

    def compact(self):
        n = torch.full((1,), -7, dtype=torch.int32, device="cuda")
        specvlm.compact_pages(self.cache, self.ref, n_used=n, d_status=self.status)
        moves, n_used = self.plain.compact(self.table)
        self.check(self.copies([(a, b, self.plain.page) for a, b in moves]))
        assert int(n) == n_used and all(r > 0 for r in self.plain.ref[:n_used])


@pytest.mark.parametrize("page", [64, 192])
@pytest.mark.parametrize("pool,batch,L,H,D,unaligned", [(40, 1, 1, 1, 64, False), (61, 3, 2, 2, 128, True), (200, 17, 3, 1, 64, False), (100, 5, 3, 4, 128, False)])
def test_branches_share_until_they_write(pool, batch, L, H, D, unaligned, page):
    s = State(pool, page, batch, 3 * page, L=L, H=H, D=D, unaligned=unaligned)
    lens = [(37 * b + 5) % (2 * page) for b in range(batch)]
    s.reserve(lens)
    s.set_lens(lens)
    s.reserve([0] * batch)                                            # nothing to do
    s.fork([b % batch for b in range(2 * batch)] + [-1, 0])           # every sequence twice, the first three times, one empty
    s.reserve([7] * len(s.lens), as_list=False)
    s.set_lens([n + 7 for n in s.lens])
    s.fork(list(range(0, len(s.lens), 2)))                            # half of them end
    s.compact()
    s.compact()                                                       # nothing moves
    s.reserve([page] * len(s.lens))
    s.release()
    s.set_lens([0] * len(s.lens))
    s.release()
    assert max(s.plain.ref) == 0


def test_last_holder_keeps_the_page():
    s = State(20, 64, 1, 256)
    s.reserve([70])
    s.set_lens([70])
    s.fork([0, 0, 0])
    s.reserve([0, 1, 0])                                              # one of three writes: a copy
    assert s.plain.ref[1] == 2
    s.reserve([1, 0, 1])                                              # the two others: one copy, the last keeps it
    assert sorted(row[1] for row in s.table) == [1, 2, 3]


def test_shared_pages_ahead_are_replaced_without_a_copy():
    """Branches of a sequence that was cut back to the middle of pages that others hold whole."""
    s = State(20, 64, 1, 256)
    s.reserve([256])
    s.set_lens([256])
    s.fork([0, 0])
    s.set_lens([70, 128])
    s.reserve([150, 64])
    assert len(set(s.table[0][1:]) & set(s.table[1][1:])) == 0 and s.table[0][0] == s.table[1][0]


def test_too_few_pages_changes_nothing():
    s = State(5, 64, 3, 256)
    assert s.reserve([100, 64, 1])                                    # four of five
    s.set_lens([100, 64, 1])
    assert not s.reserve([100, 64, 64], expect=specvlm.ERR_NO_PAGES)
    assert s.reserve([0, 64, 0])
    assert not s.reserve([0, 0, 64], expect=specvlm.ERR_NO_PAGES)
    assert s.reserve([28, 64, 63])


def test_sequences_out_of_range_get_nothing():
    s = State(30, 64, 5, 256)
    s.set_lens([250, -3, 257, 10, 0])
    s.reserve([7, 1, 0, -1, 256], expect=specvlm.ERR_INVALID_ARG)
    assert all(e == -1 for row in s.table[:4] for e in row) and min(s.table[4]) >= 0


def test_entries_outside_the_pool_are_unmapped():
    s = State(9, 64, 2, 256)
    s.table = [[9, -1, 1000, -9], [2 ** 31 - 1, -(2 ** 31), 3, 4]]
    s.plain.ref[3] = s.plain.ref[4] = 1
    s.ref.copy_(_i32(s.plain.ref))
    s._cache()
    s.set_lens([10, 0])
    s.reserve([200, 70])
    s.set_lens([210, 70])
    s.fork([1, 0])
    s.compact()


def test_bad_parents_and_lengths_are_reported():
    s = State(9, 64, 2, 256)
    s.reserve([100, 10])
    s.set_lens([100, 10])
    table, lens = torch.full((3, 4), 77, dtype=torch.int32, device="cuda"), torch.full((3,), 77, dtype=torch.int32, device="cuda")
    specvlm.fork_pages(s.cache, s.ref, _i32([1, 2, -2]), table, lens, d_status=s.status)
    assert int(s.status) == specvlm.ERR_INVALID_ARG
    assert table.tolist() == [s.table[1]] + [[-1] * 4] * 2 and lens.tolist() == [10, 0, 0]
    assert s.ref.tolist() == [0, 0, 1] + [0] * 6
    s.status.zero_()
    s = State(9, 64, 2, 256)
    s.reserve([100, 10])
    s.set_lens([-1, 300])
    specvlm.release_pages(s.cache, s.ref, d_status=s.status)
    assert int(s.status) == specvlm.ERR_INVALID_ARG and s.ref.tolist() == [1, 1, 1] + [0] * 6
    specvlm.fork_pages(s.cache, s.ref, _i32([0, 1]), torch.empty_like(s.cache.block_table), torch.empty_like(s.cache.seq_lens))
    assert s.ref.tolist() == [0] * 9


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (64, 0), (65, 64), (100, 65), (500, 3), (10 ** 6, 0), (None, 0)])
def test_release_keeps_window_and_sinks(window, sinks):
    lens = [0, 1, 63, 64, 65, 128, 129, 300, 511, 512]
    s = State(100, 64, len(lens), 600, L=1, H=1)
    s.reserve([min(600, n + 80) for n in lens])
    s.set_lens(lens)
    s.release(window, sinks)
    s.reserve([88] * len(lens))                                       # a sequence goes on behind a window's gap
    s.set_lens([n + 88 for n in lens])
    s.release(window, sinks)


@pytest.mark.parametrize("pool", [1, 15, 16, 17, 16384, 16385, 40000])
def test_pools_of_any_size(pool):
    """Rounds of the planning CTA: 16 counts a thread, 16 384 a round."""
    s = State(pool, 64, 8, 64 * 4000, L=1, H=1)
    per = pool // 8
    want = [64 * per + (64 if b < pool % 8 else 0) for b in range(8)]
    s.reserve([min(n, s.max_len) for n in want])                      # more than a round of slots, and all pages where they fit
    s.set_lens([min(n, s.max_len) for n in want])
    s.fork([7, 5, 3])
    s.compact()
    s.reserve([s.max_len - n for n in s.lens])
    s.release(64 * 50, 1)
    s.compact()


def test_rows_of_any_stride():
    """Pages that lie token by token, with room between the rows."""
    L, pool, H, page, D = 2, 7, 2, 64, 64
    store = torch.zeros((L, pool, page, H, D + 8), dtype=torch.bfloat16, device="cuda")
    k, v = (store.clone().normal_()[..., :D].permute(0, 1, 3, 2, 4) for _ in range(2))
    s = State(pool, page, 1, 256, L=L, H=H)
    s.k, s.v = k, v
    s._cache()
    s.reserve([100])
    s.set_lens([100])
    s.fork([0, 0, 0])
    s.reserve([1, 2, 3])
    s.set_lens([0, 102, 0])
    s.release()
    s.compact()


def test_capture_and_two_graphs_of_one_workspace():
    s = State(40, 64, 2, 640)
    s.reserve([70, 10])
    s.set_lens([70, 10])
    ws = torch.empty(specvlm.pages_workspace_bytes(s.cache, 2), dtype=torch.uint8, device="cuda")
    graphs = []
    for call in (lambda: specvlm.reserve_pages(s.cache, s.ref, 64, ws=ws), lambda: specvlm.compact_pages(s.cache, s.ref, ws=ws)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for i in range(3):
        graphs[0].replay()
        copies, ok, _ = s.plain.reserve(s.table, s.lens, [64, 64], 640)
        assert ok and not copies
        s.set_lens([n + 64 for n in s.lens])
        s.check()
        if i == 1:
            s.set_lens([s.lens[0], 0])
            s.release()
        pool = s.copies([(a, b, 64) for a, b in s.plain.compact(s.table)[0]])
        graphs[1].replay()
        s.check(pool)
    assert launches(lambda: specvlm.release_pages(s.cache, s.ref)) == 1


@pytest.mark.parametrize("seed", range(6))
def test_random_run_follows_every_row(seed):
    """Sequences are appended to, cut back, branched, ended, windowed and the pool compacted; each sequence's rows that it
    still has pages for read what was appended to it."""
    rng = np.random.default_rng(seed)
    page, max_len, L, H, D = (64, 128)[seed % 2], 700, 2, 2, 64
    s = State(60, page, 4, max_len, L=L, H=H, D=D, seed=seed)
    content = [[] for _ in range(4)]                                  # per sequence: an id per token
    windowed = False
    for step in range(60):
        what = rng.choice(["grow", "grow", "grow", "cut", "fork", "window", "compact"])
        if what == "grow":
            new = [int(min(rng.integers(0, 100), max_len - n)) for n in s.lens]
            if not s.reserve(new):
                s.fork([i for i in range(len(s.lens)) if i % 2 == 0] or [-1])
                content = [content[i] for i in range(0, len(content), 2)] or [[]]
                continue
            n_new = max(new)
            if n_new == 0:
                continue
            ids = rng.integers(0, 250, (len(new), n_new))
            rows = torch.from_numpy(ids).to(torch.bfloat16).cuda()[None, :, :, None, None].repeat(1, 1, 1, 1, D)
            rows = rows.expand(L, len(new), n_new, H, D)                    # the same row for all layers and heads
            rope = specvlm.Rope(torch.zeros(D // 2, dtype=torch.float64))       # no turn: the rows arrive as they are
            specvlm.rope_append_kv(s.cache, rope, None, rows, rows, new_lens=_i32(new), d_status=s.status)
            s.lens = [n + m for n, m in zip(s.lens, new)]
            for c, i, m in zip(content, ids, new):
                c.extend(i[:m].tolist())
            s.check()
        elif what == "cut":
            cut = [int(rng.integers(0, min(6, n) + 1)) for n in s.lens]
            s.set_lens([n - c for n, c in zip(s.lens, cut)])
            content = [c[:n] for c, n in zip(content, s.lens)]
        elif what == "fork":
            parents = [int(rng.integers(-1, len(s.lens))) for _ in range(int(rng.integers(1, 6)))]
            s.fork(parents)
            content = [list(content[p]) if p >= 0 else [] for p in parents]
        elif what == "window":
            s.release(int(rng.integers(100, 400)), int(rng.integers(0, 70)))
        else:
            s.compact()
        k = s.k.cpu()
        for b, c in enumerate(content):
            for j, at in enumerate(s.table[b]):
                rows = c[j * page:(j + 1) * page]
                if at >= 0 and rows:
                    assert k[0, at, 0, :len(rows), 0].int().tolist() == rows and k[L - 1, at, H - 1, :len(rows), D - 1].int().tolist() == rows
