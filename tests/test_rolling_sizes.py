"""Sizes that leave the integers that the entries count them in: refused."""
import ctypes
import os
import subprocess
import sys

import pytest

from paper_2508_16201_b200 import specvlm
from test_rolling_host import _append, _kv, _with

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("layers,batch,n_new", [(2 ** 30, 2 ** 30, 16), (2 ** 31 - 1, 2 ** 31 - 1, 256), (2 ** 30, 2 ** 29, 32), (2 ** 20, 2 ** 10, 1),
                                                (1, 2 ** 30, 1), (2 ** 22, 1, 256)])
def test_rope_append_refuses_more_tokens_than_it_counts(layers, batch, n_new):
    """In a process of its own: a division by zero ends it."""
    code = ("import sys; sys.path[:0] = [%r, %r]\nfrom test_rolling_sizes import _call\nsys.exit(0 if _call(%d, %d, %d) else 1)"
            % (HERE, os.path.join(HERE, ".."), layers, batch, n_new))
    assert subprocess.run([sys.executable, "-c", code]).returncode == 0


def _call(layers, batch, n_new):
    return _append(kv=_with(_kv, n_layers=layers), batch=batch, n_new=n_new) == specvlm.ERR_UNSUPPORTED_SHAPE


def test_page_calls_refuse_pools_that_their_counts_leave_32_bits_in():
    """The planning CTA goes through the pool 16 384 pages at a time, in 32 bits."""
    L, f = specvlm.lib(), ctypes.byref
    for pages, want in ((2 ** 30, specvlm.ERR_UNSUPPORTED_SHAPE), (2 ** 31 - 1, specvlm.ERR_UNSUPPORTED_SHAPE)):
        kv = _with(_kv, n_blocks=pages)
        assert L.specvlm_reserve_pages(f(kv), 0x2000, 0x6000, 2, 3, None, 0x10000, 1 << 62, None, None) == want
        assert L.specvlm_compact_pages(f(kv), 0x2000, 0x6000, 2, None, 0x10000, 1 << 62, None, None) == want
        assert L.specvlm_release_pages(f(kv), 0x2000, 0x6000, 2, 1, 0, None, None) == want
        assert L.specvlm_fork_pages(f(kv), 0x6000, 2, 0x7000, 2, 0x8000, 0x9000, None, None) == want
        assert L.specvlm_pages_workspace_bytes(f(kv), 2) == 0
    assert L.specvlm_pages_workspace_bytes(f(_with(_kv, n_blocks=2 ** 30 - 1)), 2) > 0
