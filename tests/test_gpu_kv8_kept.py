"""Calls over an 8-bit cache that cannot be carried out leave the cache as it was: too many sequences for an attention kernel, workspaces
that the card does not hold."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from test_gpu_kv8 import Cache, attn

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

MANY = 65536


def _state(c, ids):
    def length(i):
        try:
            return c.ctx.kv_seq_len(c.desc, i)
        except ss.SeesawError as e:
            assert e.code == ss.SS_ENOENT
            return None
    return [length(i) for i in ids], c.ctx.kv_free_pages(c.desc)


@pytest.mark.parametrize("dtype,what", [(wl.BF16, "prefill"), (wl.F32, "prefill"), (wl.F16, "decode"), (wl.F32, "decode")])
def test_more_sequences_than_attention_takes(dtype, what):
    rng = np.random.default_rng(61)
    c = Cache(dtype, 1, 1, 64, pages=MANY + 16, seqs=MANY + 2, max_len=64)
    q, k, v = (c.tokens(rng, 64, 1) for _ in range(3))
    c.ctx.kv8_write(c.desc, 0, [0], [20], [0], k[1][:20], v[1][:20])
    before = _state(c, [0, 1, 2, MANY - 1, MANY])
    held = c.export([0], [20])[0]
    ids, at = np.arange(MANY), np.zeros(MANY, dtype=np.int32)
    at[0] = 20
    n = np.ones(MANY, dtype=np.int32)
    if what == "prefill":
        n[0] = 30                                           # begins inside a block and goes on into the ones behind
    big = torch.zeros(int(n.sum()), 1, 64, device="cuda", dtype=q[1].dtype)
    big[:30] = k[1][20:50]
    with pytest.raises(ss.SeesawError) as e:
        if what == "prefill":
            c.ctx.kv8_attn_prefill(c.desc, 0, ids, n, at, big, big, big, torch.empty_like(big))
        else:
            c.ctx.kv8_attn_decode(c.desc, 0, ids, at, big, big, big, torch.empty_like(big))
    assert e.value.code == ss.SS_EINVAL
    assert _state(c, [0, 1, 2, MANY - 1, MANY]) == before
    assert np.array_equal(c.export([0], [20])[0], held)
    # without the sequence too many the same call goes through
    ids, at, n = ids[:-1], at[:-1], n[:-1]
    big = big[:int(n.sum())].contiguous()
    out = torch.empty_like(big)
    if what == "prefill":
        c.ctx.kv8_attn_prefill(c.desc, 0, ids, n, at, big, big, big, out)
    else:
        c.ctx.kv8_attn_decode(c.desc, 0, ids, at, big, big, big, out)
    torch.cuda.synchronize()
    assert _state(c, [0, 1, MANY - 2, MANY - 1])[0] == [20 + int(n[0]), 1, 1, None]
    assert np.array_equal(c.export([0], [20 + int(n[0])])[0][:, :, :16], held[:, :, :16])


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


def test_a_cache_that_the_card_does_not_hold():
    """A terabyte of pages: the call that would allocate them says so, and nothing that follows is told of it."""
    rng = np.random.default_rng(63)
    c, small = (Cache(wl.BF16, 1, 1, 64, pages=p, seqs=1) for p in (1 << 30, 4))
    k = c.tokens(rng, 5, 1)[1]
    small.ctx.kv8_write(small.desc, 0, [0], [5], [0], k, k)
    for _ in range(2):
        _out_of_memory(lambda: c.ctx.kv8_write(c.desc, 0, [0], [5], [0], k, k))
    got = attn(small, 0, [0], [5], [0], k, k, k, False)
    assert np.isfinite(got).all() and float((k + 1).sum()) == float((k + 1).sum())


def test_a_workspace_that_the_card_does_not_hold():
    c, call, one, watched = _too_large()
    before = _state(c, watched)
    for _ in range(2):
        _out_of_memory(call)
        assert _state(c, watched) == before
    a, b = one(100), one(101)
    assert np.array_equal(a, b) and np.isfinite(a).all()
    assert _state(c, watched)[0] == before[0][:2] + [32, 32]
