"""What the Python entries of the rolling cache refuse before any native call, with tensors of the host: outputs that a kernel would
write past, or write in another order than theirs."""
import pytest
import torch

from paper_2508_16201_b200 import specvlm

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class _Native:
    """Stands for the native module: keeps what it is called with, and answers that all went well."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def native(monkeypatch):
    fake = _Native()
    monkeypatch.setattr(specvlm, "native", lambda: fake)
    return fake


def _cache(seq_lens=None, paged=True):
    k = torch.zeros((2, 5, 2, 64, 64), dtype=BF16)
    table = torch.zeros((2, 2), dtype=I32) if paged else None
    return specvlm.KvCache(k, k.clone(), torch.zeros(2, dtype=I32) if seq_lens is None else seq_lens, 64, table)


def _window(q_shape=(2, 2, 3, 8, 64), **kw):
    return specvlm.window_attn(_cache(), torch.zeros(q_shape, dtype=BF16), 10, 1, 0.125, ws=torch.empty(1 << 16, dtype=torch.uint8), **kw)


def test_window_outputs_that_fit_are_taken(native):
    out, lse = torch.empty((2, 2, 3, 8, 64), dtype=BF16), torch.empty((2, 2, 3, 8), dtype=F32)
    assert _window(out=out, lse=lse) is out and _window(out=out) is out and _window(lse=lse).shape == out.shape
    assert [name for name, _ in native.calls] == ["window_attn"] * 3 and native.calls[0][1][8] is out and native.calls[0][1][9] is lse


@pytest.mark.parametrize("out", [
    torch.empty((2, 2, 1, 8, 64), dtype=BF16),                       # that of a call of one token: written past its end
    torch.empty((2, 2, 3, 8, 128), dtype=BF16)[..., :64],            # strided rows: written as if they were not
    torch.empty((2, 2, 3, 64, 8), dtype=BF16).transpose(3, 4),
    torch.empty((2, 2, 3, 8, 64), dtype=F32), torch.empty((2, 2, 3, 8, 64), dtype=torch.float16),
    torch.empty(2 * 2 * 3 * 8 * 64, dtype=BF16)])
def test_window_outputs_that_do_not_fit_are_refused(native, out):
    with pytest.raises(AssertionError):
        _window(out=out)
    assert native.calls == []


@pytest.mark.parametrize("lse", [
    torch.empty((2, 2, 1, 8), dtype=F32), torch.empty((2, 2, 3, 16), dtype=F32)[..., ::2], torch.empty((2, 2, 8, 3), dtype=F32),
    torch.empty((2, 2, 3, 8), dtype=BF16), torch.empty((2, 2, 3, 8), dtype=torch.float64), torch.empty((2, 2, 3, 8, 1), dtype=F32)])
def test_window_lse_that_does_not_fit_is_refused(native, lse):
    with pytest.raises(AssertionError):
        _window(lse=lse)
    assert native.calls == []


def test_strided_lengths_are_refused():
    """Lengths are read, and by the append written, one after the other."""
    lens = torch.zeros((2, 2), dtype=I32)
    assert _cache(lens[0]).struct.seq_lens == lens.data_ptr() and _cache(torch.zeros(4, dtype=I32)).n_seqs == 2
    for bad in (lens[:, 0], torch.zeros(1, dtype=I32).expand(2), torch.zeros(4, dtype=I32)[::2]):
        for paged in (False, True):
            with pytest.raises(AssertionError):
                _cache(bad, paged)
