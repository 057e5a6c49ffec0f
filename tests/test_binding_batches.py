"""Lists of a batch that are too short are not handed over (no GPU, nothing is called)."""
import numpy as np
import pytest

from paper_2503_06433_amd import binding as b


class _Nothing:
    def __getattr__(self, name):
        raise AssertionError("%s is called" % name)


def _context():
    c = b.Context.__new__(b.Context)
    c.h, c.lib = None, _Nothing()
    c.model, c.runtime = b.ModelCfg(256, 4, 2, 64, 64, 1, 0, 1e-5, 1e4, b.SS_BF16, 16), b.RuntimeCfg(4, 0, 0, 0, 64)
    return c


def test_a_batch_has_a_length_and_a_position_for_every_sequence():
    c = _context()
    bt, keep = c._batch([7, 8], [1, 2], [0, 3])
    assert bt.n_seqs == 2 and [list(x) for x in keep] == [[7, 8], [1, 2], [0, 3]]
    for lens, at in (([1], [0, 3]), ([1, 2], [0]), ([], [0, 3]), ([1, 2], np.zeros(1, dtype=np.int32))):
        with pytest.raises(ValueError):
            c._batch([7, 8], lens, at)


@pytest.mark.parametrize("call", [
    lambda c, d: c.layer_prefill(d, 0, 1, [1, 2], [3, 3], [0], None, None),
    lambda c, d: c.layer_prefill(d, 0, 1, [1, 2], [3], [0, 0], None, None),
    lambda c, d: c.layer_decode(d, 0, 1, [1, 2], [5], None, None),
    lambda c, d: c.layers_prefill(d, [1, 2], [3, 3], [0], None, None),
    lambda c, d: c.layers_decode(d, [1, 2], [5], None, None),
    lambda c, d: c.kv_import_dev(d, [1, 2], [5], None),
    lambda c, d: c.kv8_write(d, 0, [1, 2], [3, 3], [0], None, None),
    lambda c, d: c.kv8_attn_prefill(d, 0, [1, 2], [3], [0, 0], None, None, None, None),
    lambda c, d: c.kv8_attn_decode(d, 0, [1, 2], [5], None, None, None, None)])
def test_short_lists_are_refused_by_every_call(call):
    with pytest.raises(ValueError):
        call(_context(), b.ShardDesc(b.SS_PP, 1, 0, 0, 1))
