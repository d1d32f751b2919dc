"""The cache operators' binding: what it takes for a table of frequencies.  No device needed: an empty or a bad table is refused before CUDA is
touched, a good one comes as far as the device."""
import array

import numpy as np
import pytest

from paper_2410_15240_b200 import fastrack, kv

torch = pytest.importorskip("torch")
GOOD = [0.5 ** i for i in range(8)]


def create(frequencies, rotary=kv.ROTARY_HALF):
    """The result code of making a handle with this table."""
    try:
        kv.KvCache(kv.BF16, kv.INT8, 8, 2, 128, 64, rotary=rotary, frequencies=frequencies).close()
    except fastrack.FastrackError as e:
        return e.code
    return fastrack.OK


@pytest.mark.parametrize("kind", [list, tuple, iter, np.array, torch.tensor, lambda x: array.array("d", x), lambda x: np.array(x, np.float32)])
def test_any_sequence_of_frequencies(kind):
    reached = fastrack.OK if torch.cuda.is_available() else fastrack.ERR_CUDA
    assert create(kind(GOOD)) == reached
    assert create(kind(GOOD[:7])) == fastrack.ERR_ARG           # 14 channels: not a multiple of 16


@pytest.mark.parametrize("empty", [None, (), np.array([]), torch.tensor([])])
def test_no_frequencies(empty):
    assert create(empty) == fastrack.ERR_ARG                    # rotary without a table
    assert create(empty, kv.ROTARY_NONE) == (fastrack.OK if torch.cuda.is_available() else fastrack.ERR_CUDA)
