"""Calls over an 8-bit cache that cannot be carried out leave the cache as it was: too many sequences for an attention kernel, workspaces
that the card does not hold."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from test_gpu_kv8 import Cache, attn

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

def _too_large():
    """A cache and the arguments of a step that would keep the scores of 65472 heads over a million tokens: 340 GB of workspace.  Sequences
    100 and 101 hold the same 31 tokens."""
    heads, n_long, n = 65472, 8, 160000
    rng = np.random.default_rng(62)
    c = Cache(wl.BF16, heads, 1, 64, pages=n_long * (n // 16 + 1) + 16, seqs=n_long + 4, max_len=n + 64, weights=True)
    k = torch.randn(n, 1, 64, device="cuda").to(torch.bfloat16)
    for i in range(n_long):
        for t in range(0, n, 16000):
            c.ctx.kv8_write(c.desc, 0, [i], [16000], [t], k[t:t + 16000], k[t:t + 16000])
    short = c.tokens(rng, 40, 1)[1]
    q = torch.randn(n_long + 1, heads, 64, device="cuda").to(torch.bfloat16)
    c.ctx.kv8_write(c.desc, 0, [100, 101], [31, 31], [0, 0], *(torch.cat([short[:31], short[:31]]) for _ in range(2)))
    kv = torch.cat([k[:n_long], short[31:32]])
    call = lambda: c.ctx.kv8_attn_decode(c.desc, 0, list(range(n_long)) + [100], [n] * n_long + [31], q, kv, kv, torch.empty_like(q))
    one = lambda i: attn(c, 0, [i], None, [31], q[n_long:], short[31:32], short[31:32], True)
    return c, call, one, [0, n_long - 1, 100, 101]


def _out_of_memory(call):
    with pytest.raises(ss.SeesawError) as e:
        call()
    assert e.value.code == ss.SS_ENOMEM


def test_an_allocation_that_failed_does_not_fail_the_next_call():
    c, call, one, _ = _too_large()
    _out_of_memory(call)
    assert np.isfinite(one(101)).all()
