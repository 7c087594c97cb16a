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


@pytest.mark.parametrize("many", [2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1, 2 ** 64 + 1])
def test_more_than_any_cache_holds_is_everything(native, many):
    """A window, sinks or a number of new tokens beyond 32 bits are not taken modulo 2^32."""
    most = 2 ** 31 - 1
    cache, counts = _cache(), torch.zeros(5, dtype=I32)
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    q = torch.zeros((2, 2, 3, 8, 64), dtype=BF16)
    specvlm.window_attn(cache, q, many, many, 0.125, ws=ws)
    specvlm.release_pages(cache, counts, window=many, n_sinks=many)
    specvlm.release_pages(cache, counts, n_sinks=1)
    specvlm.reserve_pages(cache, counts, many, ws=ws)
    window, release, plain, reserve = (args for _, args in native.calls)
    assert window[5:7] == (most, most) and release[4:6] == (most, most) and plain[4:6] == (most, 1) and reserve[4] == most
    size = specvlm.window_attn_workspace_bytes(cache, 2, 8, 3, many, many)
    assert size == specvlm.window_attn_workspace_bytes(cache, 2, 8, 3, most, most) > 0


@pytest.mark.parametrize("few", [0, -1, -2 ** 31, -2 ** 32, -2 ** 32 + 5, -2 ** 40 + 1])
def test_a_window_of_nothing_stays_one(native, few):
    """... nor are negative ones: what is passed on is refused as it was."""
    cache, counts = _cache(), torch.zeros(5, dtype=I32)
    specvlm.window_attn(cache, torch.zeros((2, 2, 3, 8, 64), dtype=BF16), few, few, 0.125, ws=torch.empty(1 << 16, dtype=torch.uint8))
    specvlm.release_pages(cache, counts, window=few, n_sinks=few)
    specvlm.reserve_pages(cache, counts, few, ws=torch.empty(1 << 16, dtype=torch.uint8))
    for x in native.calls[0][1][5:7] + native.calls[1][1][4:6] + native.calls[2][1][4:5]:
        assert -2 ** 31 <= x <= 0 and (x < 0 or few == 0)
    assert specvlm.window_attn_workspace_bytes(cache, 2, 8, 3, few, 1) == 0
