"""Writes of tokens know nothing of the attention that may follow: neither its limits nor its work lists."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from oracle import kv8
from test_gpu_kv8 import Cache, attn

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_a_long_write_for_many_query_heads():
    """More (token, query head) pairs than one call of attention takes."""
    n, heads = 20000, 65472
    c = Cache(wl.BF16, heads, 1, 64, pages=2 * (n // 16 + 1), seqs=2, max_len=n)
    k, v = (torch.randn(n, 1, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    c.ctx.kv8_write(c.desc, 0, [0], [n], [0], k, v)
    for t in range(0, n, 4000):
        c.ctx.kv8_write(c.desc, 0, [1], [4000], [t], k[t:t + 4000], v[t:t + 4000])
    a, b = c.export([0, 1], [n, n])
    assert np.array_equal(a, b)
    c.same(a[0, 0][-100:], c.held(k[-(16 * 6 + n % 16 + 16):].double().cpu().numpy())[-100:])


@pytest.mark.parametrize("dtype", [wl.BF16, wl.F32])
def test_the_same_batch_written_and_then_attended_to(dtype):
    """The second call finds the first one's page lists and still has what attention needs."""
    rng = np.random.default_rng(91)
    c = Cache(dtype, 4, 2, 64)
    lens, ids = [70, 5, 33], [2, 0, 9]
    q, k, v = (c.tokens(rng, sum(lens), h) for h in (4, 2, 2))
    for _ in range(2):
        c.ctx.kv8_write(c.desc, 0, ids, lens, [0] * 3, k[1], v[1])
        got = attn(c, 0, ids, lens, [0] * 3, q[1], k[1], v[1], False)
        t = 0
        for n in lens:
            ref, mag, _ = kv8.attention(q[0][t:t + n], c.held(k[0][t:t + n]), c.held(v[0][t:t + n]), 0)
            c.close(got[t:t + n], ref, mag)
            t += n


def test_many_new_sequences_at_once():
    """A quarter of a million of them; one that is there twice is found wherever it stands."""
    n = 1 << 18
    c = Cache(wl.BF16, 1, 1, 64, pages=n, seqs=n, max_len=16)
    k = torch.randn(n, 1, 64, device="cuda").to(torch.bfloat16)
    ids, one, none = np.random.default_rng(92).permutation(n) * 7 - 5, np.ones(n, dtype=np.int32), np.zeros(n, dtype=np.int32)
    for a, b in ((0, n - 1), (n // 2, n // 3), (n - 2, n - 1)):
        twice = ids.copy()
        twice[a] = twice[b]
        with pytest.raises(ss.SeesawError) as e:
            c.ctx.kv8_write(c.desc, 0, twice, one, none, k, k)
        assert e.value.code == ss.SS_EINVAL and c.ctx.kv_free_pages(c.desc) == n
    c.ctx.kv8_write(c.desc, 0, ids, one, none, k, k)
    assert c.ctx.kv_free_pages(c.desc) == 0
    got = c.export(ids[-9:], [1] * 9)
    for x, y in zip(got, k[-9:].double().cpu().numpy()):
        assert np.array_equal(x[0, 0, 0], y) and np.array_equal(x[0, 1, 0], y)
