"""What the binding hands to the library: id lists and rows of tokens (no GPU, nothing is called)."""
import numpy as np
import pytest
import torch

from paper_2503_06433_amd import binding as b


@pytest.mark.parametrize("make", [b._i64, b._i32])
@pytest.mark.parametrize("given", [[], [7], [3, -1, 5], (1, 2), np.arange(6), np.arange(12)[::2], np.arange(5, dtype=np.int16)])
def test_lists_arrive_whole(make, given):
    a = make(given)
    p = b._p(a)
    assert [p[i] for i in range(len(given))] == [int(x) for x in given]


def test_read_only_arrays_are_taken():
    a = np.arange(4, dtype=np.int64)
    a.flags.writeable = False
    p = b._p(b._i64(a))
    assert [p[i] for i in range(4)] == [0, 1, 2, 3]


def test_rows_of_tokens():
    t = torch.zeros(5, 12, 16)
    at = t.data_ptr()
    assert b._rows(None, 192) == (None, 0)
    assert b._rows(t, 192) == (at, 192)
    assert b._rows(t.view(5, 192), 192) == (at, 192)
    assert b._rows(t[:, 4:8], 64) == (at + 4 * 4 * 16, 192)          # a part of a fused row
    assert b._rows(t[:, :1], 16) == (at, 192)
    assert b._rows(t[::2], 192) == (at, 384)
    assert b._rows(t[3:4, :4], 64)[1] == 64                          # one token: no stride to speak of
    assert b._rows(torch.zeros(5, 1, 16).expand(5, 1, 16), 16)[1] == 16


@pytest.mark.parametrize("make", [lambda t: t[:, ::2], lambda t: t.transpose(1, 2), lambda t: t[:, :, :8], lambda t: t[:, :, ::2],
                                  lambda t: t[:, :1].expand(5, 12, 16), lambda t: t[:, :, :1].expand(5, 12, 16)])
def test_rows_with_gaps_are_refused(make):
    t = make(torch.zeros(5, 12, 16))
    with pytest.raises(ValueError):
        b._rows(t, t[0].numel())


def test_rows_of_another_width_are_refused():
    with pytest.raises(ValueError):
        b._rows(torch.zeros(5, 12, 16), 191)
