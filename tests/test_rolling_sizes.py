"""Sizes whose product leaves 64 bits: refused by the C entries, which once divided by the number of tokens that was left of it."""
import subprocess
import sys
import os

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
