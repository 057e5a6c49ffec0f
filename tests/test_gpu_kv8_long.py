"""The 8-bit cache where its kernels share work out: prompts whose keys are cut into parts, steps whose caches many waves read, evictions
that keep a few tokens of many pages or read more keys than are held on chip, and values at the ends of the type's range.  Against
the statement in 64 bits, with the tolerances of the short cases: they do not grow with the length (a sum of weights has fp32's 2^-24
of rounding for every factor of two in it, 2^-20 for a million tokens; the joins of parts add one each)."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from oracle import kv8
from test_gpu_kv8 import Cache, attn

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype,n_q,n_kv,d", [(wl.BF16, 8, 1, 128), (wl.F16, 2, 2, 128), (wl.F16, 12, 2, 64), (wl.BF16, 1, 1, 64)],
                         ids=["bf16-8over1-128", "f16-2over2-128", "f16-12over2-64", "bf16-1over1-64"])
def test_chunks_behind_long_caches(dtype, n_q, n_kv, d):
    """One token to several hundred behind caches of 1024 to 3000, from aligned and unaligned places, and one long prompt; the last
    value of one sequence, in its open block, is infinite."""
    rng = np.random.default_rng(31)
    c = Cache(dtype, n_q, n_kv, d, pages=900, max_len=4096)
    old, new = [2999, 1024, 1500, 1040, 0], [1, 64, 300, 259, 1300]
    seqs = [[c.tokens(rng, a + b, n_q, 2.0), c.tokens(rng, a + b, n_kv), c.tokens(rng, a + b, n_kv)] for a, b in zip(old, new)]
    ids = [4, 9, 0, 2, 7]
    v3 = seqs[3][2][1].clone()
    v3[-1, 0, 5] = float("inf")
    have = [i for i in range(5) if old[i]]
    part = lambda j, i, lo, hi: (v3 if (i, j) == (3, 2) else seqs[i][j][1])[lo:hi]
    c.ctx.kv8_write(c.desc, 0, [ids[i] for i in have], [old[i] for i in have], [0] * len(have),
                    *(torch.cat([part(j, i, 0, old[i]) for i in have]) for j in (1, 2)))
    q, k, v = (torch.cat([part(j, i, old[i], old[i] + new[i]) for i in range(5)]) for j in range(3))
    first = attn(c, 0, ids, new, old, q, k, v, False)
    again = attn(c, 0, ids, new, old, q, None, None, False)
    np.testing.assert_array_equal(first, again)
    t = 0
    for i in range(5):
        kk, vv = (c.held(seqs[i][j][0]) for j in (1, 2))
        ref, mag, _ = kv8.attention(seqs[i][0][0][old[i]:], kk, vv, old[i])
        n = new[i] - (i == 3)                                    # its last query sees the infinite value
        c.close(first[t:t + n], ref[:n], mag[:n])
        if i == 3:
            assert np.isnan(first[t + n, :n_q // n_kv]).all()
        t += new[i]
    # a piece of a long cache in the middle, alone
    got = attn(c, 0, [7], [17], [1200], seqs[4][0][1][1200:1217], None, None, False)
    kk, vv = (c.held(seqs[4][j][0]) for j in (1, 2))
    ref, mag, _ = kv8.attention(seqs[4][0][0][1200:1217], kk, vv, 1200)
    c.close(got, ref, mag)


@pytest.mark.parametrize("dtype,n_q,n_kv,d", [(wl.BF16, 8, 1, 128), (wl.F16, 4, 4, 64), (wl.F32, 2, 1, 64)],
                         ids=["bf16-8over1-128", "f16-4over4-64", "f32-2over1-64"])
def test_steps_over_long_caches(dtype, n_q, n_kv, d):
    rng = np.random.default_rng(32)
    c = Cache(dtype, n_q, n_kv, d, pages=1000, max_len=9100, weights=True)
    lens = [3, 1151, 1168, 2600, 9007]
    s = [[c.tokens(rng, n, n_q, 2.0), c.tokens(rng, n, n_kv), c.tokens(rng, n, n_kv)] for n in lens]
    ids = list(range(len(lens)))
    c.ctx.kv8_write(c.desc, 0, ids, [n - 1 for n in lens], [0] * len(lens), *(torch.cat([x[j][1][:-1] for x in s]) for j in (1, 2)))
    got = attn(c, 0, ids, None, [n - 1 for n in lens], *(torch.cat([x[j][1][-1:] for x in s]) for j in range(3)), True)
    buf = torch.full((n_kv * sum(lens),), -1.0, device="cuda")
    c.ctx.kv8_weights(c.desc, ss.SS_OUT, ids, buf)
    w, t = buf.double().cpu().numpy(), 0
    for i, (x, n) in enumerate(zip(s, lens)):
        ref, mag, ww = kv8.attention(x[0][0][-1:], c.held(x[1][0]), c.held(x[2][0]), n - 1)
        c.close(got[i:i + 1], ref, mag)
        np.testing.assert_allclose(w[t:t + n_kv * n].reshape(n_kv, n), ww[0].reshape(n_kv, -1, n).sum(1), rtol=2.0 ** -12, atol=1e-12)
        t += n_kv * n


def _evicted(c, toks, w, keep, recent):
    """Imports, evicts, compares the cache and its weights."""
    lens = [k[0].shape[0] for k, _ in toks]
    ids, ends = list(range(len(lens))), [min(n, m) for n, m in zip(lens, keep)]
    c.ctx.kv_import_dev(c.desc, ids, lens, torch.cat([x[1].permute(1, 0, 2).reshape(-1) for s in toks for x in s]))
    c.ctx.kv8_weights(c.desc, ss.SS_IN, ids, torch.from_numpy(np.concatenate([x.reshape(-1) for x in w])).cuda())
    c.ctx.kv8_evict(c.desc, ids, keep, recent)
    buf = torch.empty(c.n_kv * sum(ends), device="cuda")
    c.ctx.kv8_weights(c.desc, ss.SS_OUT, ids, buf)
    got_w, t = buf.cpu().numpy(), 0
    store = lambda x: wl.round_to_storage(x, c.dtype)
    for i, got in enumerate(c.export(ids, ends)):
        k, v, kw = kv8.evict(*(kv8.units(x[0], c.dtype == wl.F32) for x in toks[i]), w[i], keep[i], recent, store, c.dtype == wl.F32)
        np.testing.assert_array_equal(got_w[t:t + kw.size].reshape(kw.shape), kw)
        c.same(got[0, 0], k)
        c.same(got[0, 1], v)
        t += kw.size


@pytest.mark.parametrize("dtype,n_kv,d", [(wl.BF16, 2, 128), (wl.F16, 1, 64), (wl.F32, 1, 128), (wl.F32, 2, 64)])
def test_eviction_of_all_but_a_few(dtype, n_kv, d):
    """A block of sixteen pages' tokens, of one page's, and everything between; budgets that end inside a block, below a block and
    below the newest that are asked for."""
    rng = np.random.default_rng(33)
    c = Cache(dtype, n_kv, n_kv, d, pages=1200, weights=True, max_len=8192)
    lens, keep = [7013, 3000, 2000, 333, 700], [64, 100, 1999, 5, 160]
    toks = [(c.tokens(rng, n, n_kv), c.tokens(rng, n, n_kv)) for n in lens]
    w = [rng.exponential(size=(n_kv, n)).astype(np.float32) for n in lens]
    w[4] = np.repeat(rng.permutation(700 // 4).astype(np.float32), 4)[None].repeat(n_kv, 0)      # runs of equal weight
    _evicted(c, toks, w, keep, 8)


def test_eviction_reads_keys_that_do_not_fit_on_chip():
    rng = np.random.default_rng(34)
    c = Cache(wl.F16, 1, 1, 64, pages=2600, seqs=2, weights=True, max_len=41000)
    n = 40003
    toks = [(c.tokens(rng, n, 1), c.tokens(rng, n, 1))]
    w = np.round(rng.exponential(size=(1, n)) * 64).astype(np.float32) / 64                      # some hundred values: ties
    _evicted(c, toks, [w], [300], 40)


@pytest.mark.parametrize("d", [64, 128])
def test_eviction_of_extreme_values(d):
    """Blocks from 2^-120 to 2^127, of zeros, and with values that are not finite, in full blocks and in the open one."""
    rng = np.random.default_rng(35)
    c = Cache(wl.BF16, 2, 2, d, pages=300, weights=True)
    lens, keep = [1003, 1003, 200], [500, 90, 100]
    toks = []
    for i, n in enumerate(lens):
        pair = []
        for part in range(2):
            vals, t = c.tokens(rng, n, 2)
            e = np.repeat(rng.integers(-120, 121, size=(n // 16 + 1, 2)), 16, axis=0)[:n]
            e[:, 1] = np.where(rng.random(n) < 0.2, 0, e[:, 1])
            x = np.clip(vals * 2.0 ** e[:, :, None], -3e38, 3e38)
            x[64:80] = 0
            x[300:340, 1] = 0
            x = x.astype(np.float32).astype(np.float64)
            x, raw = wl.quantize(x, wl.BF16)
            t = torch.from_numpy(raw.view(np.int16)).cuda().view(torch.bfloat16)
            if i == 2:
                x, t = x.copy(), t.clone()
                for at, g, v in ((50, 0, np.nan), (100, 1, np.inf), (198, part, -np.inf)):
                    x[at, g, 3] = v
                    t[at, g, 3] = float(v)
            pair.append((x, t))
        toks.append(tuple(pair))
    w = [rng.exponential(size=(2, n)).astype(np.float32) for n in lens]
    _evicted(c, toks, w, keep, 20)


def test_pages_beyond_4_gb():
    """The same calls in a small cache and in one whose first 65 600 pages (4.3 GB of K, as much of V) are taken: the same bits."""
    rng = np.random.default_rng(36)
    heads, d, n, taken = 32, 128, 1190, 65600
    small = Cache(wl.BF16, heads, heads, d, pages=90, seqs=4, weights=True)
    large = Cache(wl.BF16, heads, heads, d, pages=taken + 90, seqs=300, weights=True)
    fill = torch.ones(16 * 4096, heads, d, device="cuda", dtype=torch.bfloat16)
    left, first = taken, 1000
    while left:
        seqs = [min(256, left - 256 * i) for i in range(16) if left > 256 * i]                   # pages, 4096 tokens at most
        t = 16 * sum(seqs)
        large.ctx.kv8_write(large.desc, 0, list(range(first, first + len(seqs))), [16 * p for p in seqs], [0] * len(seqs), fill[:t], fill[:t])
        left -= sum(seqs)
        first += len(seqs)
    del fill
    q, k, v = (small.tokens(rng, n + 2, heads)[1] for _ in range(3))
    res = []
    for c in (small, large):
        got = [attn(c, 0, [1], [n], [0], q[:n], k[:n], v[:n], False)]
        got += [attn(c, 0, [1], None, [n + i], q[n + i:n + i + 1], k[n + i:n + i + 1], v[n + i:n + i + 1], True) for i in range(2)]
        w = torch.full((heads * (n + 2),), -1.0, device="cuda")
        c.ctx.kv8_weights(c.desc, ss.SS_OUT, [1], w)
        got += [w.cpu().numpy(), c.export([1], [n + 2])[0]]
        c.ctx.kv8_evict(c.desc, [1], [300], 30)
        got.append(c.export([1], [300])[0])
        res.append(got)
    assert large.ctx.kv_page_table(large.desc, 1).min() >= taken
    for a, b in zip(*res):
        assert np.isfinite(a).all()
        np.testing.assert_array_equal(a, b)
