"""Reservations of more slots, and of more sequences, than one pass of the planning CTA's threads takes (1024 slots a round, 32
sequences a warp), with pages that are begun, shared and have to be copied."""
import pytest
import torch

from paper_2508_16201_b200 import specvlm
from test_gpu_pages import State

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("parents", [[0, 0, 0, 1, 1, 2], [2, 1, 0, 0, 1, 1], [0] * 6])
@pytest.mark.parametrize("page", [64, 128])
def test_begun_pages_in_every_round(parents, page):
    """Six branches of three sequences that end within a page; 300 pages each, so that the first slots of the fifth and sixth, which share
    a begun page with an earlier one, come in the second round.  The copies' rows and every count follow the plain statement."""
    s = State(2000, page, 3, 304 * page, H=1, L=1)
    lens = [page + 36, 6, 3 * page + 1]
    s.reserve(lens)
    s.set_lens(lens)
    s.fork(parents)
    assert max(s.plain.ref) > 1
    before = list(s.plain.ref)
    new = [300 * page - 1, 300 * page, 299 * page + 5, 300 * page, 301 * page - 7, 250 * page]
    assert s.reserve(new) and s.plain.ref != before
    s.set_lens([n + m for n, m in zip(s.lens, new)])
    s.release(40 * page, 1)
    s.compact()


def test_shared_pages_ahead_in_every_round():
    """Branches that were cut back: pages that others hold whole lie on either side of the border of a round, and are replaced."""
    page = 64
    s = State(4000, page, 1, 700 * page, H=1, L=1)
    s.reserve([650 * page - 3])
    s.set_lens([650 * page - 3])
    s.fork([0, 0, 0])
    s.set_lens([10 * page + 1, 5 * page, 300 * page + 63])
    assert s.reserve([600 * page, 640 * page, 399 * page])           # 600 + 640 + 400 slots
    assert len({at for row in s.table for at in row if at >= 0}) > 1600
    s.set_lens([n + m for n, m in zip(s.lens, [600 * page, 640 * page, 399 * page])])
    s.compact()


def test_too_few_pages_in_the_second_round_change_nothing():
    page = 64
    s = State(1500, page, 2, 1000 * page, H=1, L=1)
    s.reserve([page + 1, 1])
    s.set_lens([page + 1, 1])
    s.fork([0, 0, 1, 1])
    assert not s.reserve([500 * page, 300 * page, 400 * page, 400 * page], expect=specvlm.ERR_NO_PAGES)
    assert not s.reserve([500 * page, 300 * page, 400 * page, 297 * page], expect=specvlm.ERR_NO_PAGES)
    # all that are free: 500, 300 and 400 ahead, a copy of either begun page, and the rest for the last
    rest = s.plain.ref.count(0) - (500 + 300 + 400 + 2)
    assert s.reserve([500 * page, 300 * page, 400 * page, rest * page])
    assert s.plain.ref.count(0) == 0


@pytest.mark.parametrize("batch,L,H", [(40, 2, 8), (40, 1, 1)])
def test_both_forms_of_the_plan(batch, L, H):
    """Copies of more than 4 MiB move in a kernel of their own, the others within the plan's cluster."""
    page = 64
    s = State(batch * 32, page, 4, 40 * page, L=L, H=H)
    lens = [page + 7, 2 * page + 63, 1, 30]
    s.reserve(lens)
    s.set_lens(lens)
    s.fork([b * b % 4 if b % 7 else 2 for b in range(batch)])
    new = [27 * page + 13 * b % 90 for b in range(batch)]                # more than 1024 slots
    assert s.reserve(new)
    s.set_lens([n + m for n, m in zip(s.lens, new)])
    s.compact()


@pytest.mark.parametrize("batch", [33, 300, 1023, 1024])
def test_batches_of_every_size(batch):
    """Every warp of the planning CTA has sequences: some without new tokens, some out of range, many that share a begun page."""
    page = 64
    s = State(4 * batch + 200, page, 50, 4 * page, H=1, L=1)
    lens = [(37 * b + 5) % (2 * page) for b in range(50)]
    s.reserve(lens)
    s.set_lens(lens)
    s.fork([(7 * b) % 50 if b % 11 else -1 for b in range(batch)])
    new = [(b * 5) % 70 for b in range(batch)]
    assert s.reserve(new)
    s.set_lens([n + m for n, m in zip(s.lens, new)])
    lens, out = list(s.lens), [4 * page + 1 if b % 97 == 3 else n for b, n in enumerate(s.lens)]
    s.set_lens(out)
    assert s.reserve([3] * batch, as_list=False, expect=specvlm.ERR_INVALID_ARG if out != lens else 0)
    s.set_lens(lens)
    s.release(60, 3)
    s.compact()
    table = torch.tensor(s.table)
    used = torch.bincount(table[table >= 0].flatten(), minlength=len(s.plain.ref))
    assert used.tolist() == s.plain.ref                               # counts and table agree
