"""Buffers of the accumulated weights that are too short, of another type, or elsewhere are refused before anything is launched."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from test_gpu_kv8 import Cache

torch = pytest.importorskip("torch")


class _Counts:
    """A library whose sequences have ten weights, and whose calls must not be reached."""
    def ss_kv8_weights_len(self, h, desc, ids, n, out):
        out._obj.value = 10
        return 0


@pytest.mark.parametrize("buf", [torch.zeros(10), torch.zeros(9), torch.zeros(10, dtype=torch.bfloat16), torch.zeros(20)[::2], np.zeros(10, dtype=np.float32)])
def test_buffers_that_do_not_fit(buf):
    from paper_2503_06433_amd import binding as b
    c = b.Context.__new__(b.Context)
    c.h, c.lib, c.runtime = None, _Counts(), b.RuntimeCfg(4, 0, 0, 0, 64)
    with pytest.raises(ValueError):
        c.kv8_weights(b.ShardDesc(b.SS_PP, 1, 0, 0, 1), ss.SS_OUT, [3], buf)


def test_calls_without_a_context_are_refused():
    assert ss.load_library().ss_kv8_weights_len(None, None, None, 0, None) == ss.SS_EINVAL


@pytest.mark.gpu
def test_buffers_of_weights():
    rng = np.random.default_rng(95)
    c = Cache(wl.BF16, 4, 2, 64, layers=2, weights=True)
    k = c.tokens(rng, 30, 2)[1]
    for layer in range(2):
        c.ctx.kv8_write(c.desc, layer, [5, 6], [20, 10], [0, 0], k, k)
    n = 2 * 2 * 30
    for bad in (torch.zeros(n - 1, device="cuda"), torch.zeros(n, device="cuda", dtype=torch.float16), torch.zeros(2 * n, device="cuda")[::2],
                torch.zeros(n), torch.zeros(0, device="cuda"), torch.zeros(n, device="cuda", dtype=torch.int32)):
        for direction in (ss.SS_IN, ss.SS_OUT):
            with pytest.raises(ValueError):
                c.ctx.kv8_weights(c.desc, direction, [5, 6], bad)
    with pytest.raises(ss.SeesawError) as e:
        c.ctx.kv8_weights(c.desc, ss.SS_OUT, [5, 7], torch.zeros(n, device="cuda"))
    assert e.value.code == ss.SS_ENOENT
    w = torch.rand(n + 3, device="cuda")                    # room for more is no fault, and stays as it is
    got = torch.full((n + 3,), 7.0, device="cuda")
    c.ctx.kv8_weights(c.desc, ss.SS_IN, [5, 6], w)
    c.ctx.kv8_weights(c.desc, ss.SS_OUT, [5, 6], got)
    assert torch.equal(got[:n], w[:n]) and (got[n:] == 7).all()
    c.ctx.kv8_weights(c.desc, ss.SS_OUT, [], torch.zeros(0, device="cuda"))
