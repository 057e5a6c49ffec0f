"""The 8-bit cache on the GPU against its statement in 64 bits (oracle/kv8.py): write, export and import, attention of single
tokens and prompts, accumulated weights, eviction, and what is refused.

Tolerances.  What a full block stands for is q * (A / 127): exact whole numbers, one fp32 product, one rounding to the model's
type: half a step of the type, relative (H below), and 2^-22 for the product.  Attention rounds the weights (relative H each, so
H times the sum of the weights times |v|), the output once (H) and forms scores, exponentials and sums in fp32: scores of
up to 40 from 128 products are off by at most 2^-24 * 128 * 40 / 16 < 2^-15, the exponential by as much relatively, and weights in
the half type below its normal range by 2^-25 of the largest each: 2^-11 of the magnitude sum covers all of it for
the 16-bit types; fp32 has no rounded weights, 2^-13 covers the scores."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from oracle import kv8

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {wl.F32: torch.float32, wl.BF16: torch.bfloat16, wl.F16: torch.float16}
H = {wl.F32: 2.0 ** -24, wl.BF16: 2.0 ** -8, wl.F16: 2.0 ** -11}
# the half type's numbers below 2^-14 are 2^-24 apart: rounding moves an output by 2^-25 there, whatever its size (a sum of
# weights of 1e-9 and values of zero is such an output); the others' lie below the 1e-30 of the bound
TINY = {wl.F32: 1e-30, wl.BF16: 1e-30, wl.F16: 2.0 ** -25 * (1 + 2.0 ** -10)}
SLACK = {wl.F32: 2.0 ** -13, wl.BF16: 2.0 ** -11, wl.F16: 2.0 ** -11}


class Cache:
    """A context with one 8-bit shard, and what its cache is to hold."""

    def __init__(self, dtype, n_q, n_kv, d, pages=400, layers=1, seqs=64, weights=False, max_len=4096, k=1, shard=0):
        self.dtype, self.n_q, self.n_kv, self.d, self.layers = dtype, n_q // k, n_kv // k, d, layers
        self.ctx = ss.Context(ss.ModelCfg(n_q * d, n_q, n_kv, d, 64, layers, 0, 1e-5, 10000.0, dtype, 16),
                              ss.RuntimeCfg(pages, 0, 0, 0, max_len))
        self.desc = ss.ShardDesc(ss.SS_TP, k, shard, 0, layers) if k > 1 else ss.ShardDesc(ss.SS_PP, 1, 0, 0, layers)
        self.ctx.kv8_enable(self.desc, seqs, weights)

    def tokens(self, rng, n, heads, scale=1.0):
        """[n, heads, d]: values of the type, in float64 and on the device."""
        x = rng.normal(size=(n, heads, self.d)) * np.exp(0.5 * rng.normal(size=(n, heads, 1))) * scale
        vals, raw = wl.quantize(x, self.dtype)
        t = torch.from_numpy(raw if self.dtype == wl.F32 else raw.view(np.int16)).cuda()
        return vals, t if self.dtype == wl.F32 else t.view(TYPES[self.dtype])

    def held(self, x):
        return kv8.held(x)

    def export(self, ids, lens):
        """[layer][K | V][tokens, heads, d] per sequence, float64."""
        out = torch.full((2 * self.layers * self.n_kv * self.d * sum(lens),), 7.0, device="cuda", dtype=TYPES[self.dtype])
        self.ctx.kv_export_dev(self.desc, ids, out)
        torch.cuda.synchronize()
        flat, at, res = out.double().cpu().numpy(), 0, []
        for n in lens:
            m = 2 * self.layers * self.n_kv * n * self.d
            res.append(flat[at:at + m].reshape(self.layers, 2, self.n_kv, n, self.d).transpose(0, 1, 3, 2, 4))
            at += m
        return res

    def same(self, got, ref):
        """Rounded once from `ref`."""
        assert got.shape == ref.shape
        np.testing.assert_array_equal(np.isnan(got), np.isnan(ref))
        bad = np.abs(got - ref) > (H[self.dtype] + 2.0 ** -22) * np.abs(ref) + TINY[self.dtype]
        assert not bad[~np.isnan(ref)].any(), (got[bad][:4], ref[bad][:4])

    def close(self, got, ref, mag):
        assert got.shape == ref.shape and np.isfinite(got).all()
        bound = H[self.dtype] * (np.abs(ref) + mag) + SLACK[self.dtype] * mag + TINY[self.dtype]
        worst = np.max(np.abs(got - ref) / bound)
        assert worst <= 1, "off by %.2f of the bound" % worst


def attn(c, layer, ids, lens, before, q, k, v, decode):
    out = torch.full((q.shape[0], c.n_q, c.d), 3.0, device="cuda", dtype=q.dtype)
    if decode:
        c.ctx.kv8_attn_decode(c.desc, layer, ids, before, q, k, v, out)
    else:
        c.ctx.kv8_attn_prefill(c.desc, layer, ids, lens, before, q, k, v, out)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


HEADS = [(wl.BF16, 4, 4, 128), (wl.F16, 8, 1, 128), (wl.BF16, 16, 2, 64), (wl.F16, 3, 3, 64), (wl.F32, 4, 2, 64), (wl.F32, 2, 1, 128),
         (wl.BF16, 20, 1, 128), (wl.F16, 40, 2, 64), (wl.BF16, 14, 2, 128)]
IDS = ["%s-%dover%d-%d" % ({0: "f32", 1: "bf16", 2: "f16"}[t], a, b, d) for t, a, b, d in HEADS]


@pytest.mark.parametrize("dtype,n_q,n_kv,d", HEADS, ids=IDS)
def test_written_in_pieces_the_cache_holds_the_same(dtype, n_q, n_kv, d):
    """One call, pieces of odd sizes, token by token: what the cache stands for depends on the tokens alone."""
    rng = np.random.default_rng(5)
    c = Cache(dtype, n_q, n_kv, d)
    lens = [1, 15, 16, 17, 33, 70, 128]
    toks = [(c.tokens(rng, n, n_kv), c.tokens(rng, n, n_kv)) for n in lens]
    cat = lambda part: torch.cat([t[part][1] for t in toks])
    ids = list(range(len(lens)))
    c.ctx.kv8_write(c.desc, 0, ids, lens, [0] * len(lens), cat(0), cat(1))
    one = c.export(ids, lens)
    for (k, v), got in zip(toks, one):
        c.same(got[0, 0], c.held(k[0]))
        c.same(got[0, 1], c.held(v[0]))
    for step in (1, 5, 16, 23):
        other = [100 * step + i for i in ids]
        done = [0] * len(lens)
        while any(a < n for a, n in zip(done, lens)):
            live = [i for i in ids if done[i] < lens[i]]
            cut = [min(step, lens[i] - done[i]) for i in live]
            part = lambda p: torch.cat([toks[i][p][1][done[i]:done[i] + m] for i, m in zip(live, cut)])
            c.ctx.kv8_write(c.desc, 0, [other[i] for i in live], cut, [done[i] for i in live], part(0), part(1))
            for i, m in zip(live, cut):
                done[i] += m
        for got, ref in zip(c.export(other, lens), one):
            assert np.array_equal(got, ref), step
        c.ctx.kv_free(c.desc, other)


def test_import_holds_what_a_write_holds_and_layers_stay_apart():
    rng = np.random.default_rng(6)
    c = Cache(wl.BF16, 8, 4, 128, layers=3, k=2, shard=1)
    lens = [5, 48, 31]
    toks = [[(c.tokens(rng, n, 2), c.tokens(rng, n, 2)) for _ in range(3)] for n in lens]
    stage = torch.cat([x[1].permute(1, 0, 2).reshape(-1) for seq in toks for layer in seq for x in layer])
    c.ctx.kv_import_dev(c.desc, [1, 2, 3], lens, stage)
    for layer in range(3):
        c.ctx.kv8_write(c.desc, layer, [11, 12, 13], lens, [0, 0, 0], torch.cat([s[layer][0][1] for s in toks]),
                        torch.cat([s[layer][1][1] for s in toks]))
    a, b = c.export([1, 2, 3], lens), c.export([11, 12, 13], lens)
    for x, y, seq in zip(a, b, toks):
        assert np.array_equal(x, y)
        for layer in range(3):
            c.same(x[layer, 0], c.held(seq[layer][0][0]))
            c.same(x[layer, 1], c.held(seq[layer][1][0]))
    raw = c.ctx.kv_read(c.desc, 12, 2, 2)
    assert np.array_equal(wl.bf16_to_f32(raw).astype(np.float64), b[1][2].transpose(0, 2, 1, 3))


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16, wl.F16])
def test_blocks_of_zeros_of_extreme_values_and_of_values_that_are_not_finite(dtype):
    rng = np.random.default_rng(7)
    c = Cache(dtype, 2, 2, 64)
    n = 16 * 6 + 3
    k, _ = c.tokens(rng, n, 2)
    k[0:16] = 0
    k[16:32] *= 1e-3 if dtype == wl.F16 else 1e-36
    k[32:48] = np.sign(k[32:48]) * (60000.0 if dtype == wl.F16 else 3e38)
    k[48, 0, 5] = np.nan                        # head 0 alone
    k[66, 1, 0] = -np.inf
    k[n - 1, 0, 0] = np.inf                     # in the open block: as it is
    with np.errstate(over="ignore"):
        vals, raw = wl.quantize(k, dtype)
    t = torch.from_numpy(raw if dtype == wl.F32 else raw.view(np.int16)).cuda()
    t = t if dtype == wl.F32 else t.view(TYPES[dtype])
    c.ctx.kv8_write(c.desc, 0, [0], [n], [0], t, t.flip(1).contiguous())
    got = c.export([0], [n])[0][0]
    for x, ref in ((got[0], c.held(vals)), (got[1], c.held(vals[:, ::-1]))):
        fin = np.isfinite(ref)
        assert np.array_equal(np.isnan(x), np.isnan(ref)) and np.array_equal(x[n - 1], ref[n - 1])
        # the smallest steps are below the normal range of fp32: one of its smallest numbers on top
        assert np.all(np.abs(x[fin] - ref[fin]) <= (H[dtype] + 2.0 ** -22) * np.abs(ref[fin]) + (2.0 ** -25 if dtype == wl.F16 else 2e-42 * 127 + 1e-40))


@pytest.mark.parametrize("dtype,n_q,n_kv,d", HEADS, ids=IDS)
def test_prompts(dtype, n_q, n_kv, d):
    """Ragged prompts from one token on, then chunks behind what is cached, from aligned and unaligned places."""
    rng = np.random.default_rng(8)
    c = Cache(dtype, n_q, n_kv, d)
    first, then = [1, 16, 33, 150, 300], [40, 1, 129, 7, 90]
    seqs = []
    for a, b in zip(first, then):
        seqs.append([c.tokens(rng, a + b, n_q, 2.0), c.tokens(rng, a + b, n_kv), c.tokens(rng, a + b, n_kv)])
    ids = [10, 3, 7, 8, 1]
    done = [0] * len(ids)
    for lens in (first, then):
        part = lambda j: torch.cat([s[j][1][o:o + n] for s, o, n in zip(seqs, done, lens)])
        got = attn(c, 0, ids, lens, done, part(0), part(1), part(2), False)
        t = 0
        for s, o, n in zip(seqs, done, lens):
            k, v = (c.held(s[j][0][:o + n]) for j in (1, 2))
            ref, mag, _ = kv8.attention(s[0][0][o:o + n], k, v, o)
            c.close(got[t:t + n], ref, mag)
            t += n
        done = [o + n for o, n in zip(done, lens)]
    # the same queries again, nothing written: also in the middle of what is cached
    at = [0, 5, 100, 40, 200]
    n = [3, 12, 62, 100, 190]
    q = torch.cat([s[0][1][a:a + m] for s, a, m in zip(seqs, at, n)])
    got, t = attn(c, 0, ids, n, at, q, None, None, False), 0
    for s, a, m, end in zip(seqs, at, n, done):
        k, v = (c.held(s[j][0][:end]) for j in (1, 2))
        ref, mag, _ = kv8.attention(s[0][0][a:a + m], k, v, a)
        c.close(got[t:t + m], ref, mag)
        t += m


@pytest.mark.parametrize("dtype,n_q,n_kv,d", HEADS, ids=IDS)
def test_single_tokens(dtype, n_q, n_kv, d):
    """Steps that open, fill and close blocks, over caches of one token to hundreds, with the weights they leave."""
    rng = np.random.default_rng(9)
    c = Cache(dtype, n_q, n_kv, d, weights=True)
    lens = [0, 1, 14, 15, 16, 31, 63, 64, 300, 777]
    steps = 3
    seqs = [[c.tokens(rng, n + steps, n_q, 2.0), c.tokens(rng, n + steps, n_kv), c.tokens(rng, n + steps, n_kv)] for n in lens]
    ids = list(range(len(lens)))
    some = [i for i in ids if lens[i]]
    c.ctx.kv8_write(c.desc, 0, some, [lens[i] for i in some], [0] * len(some), torch.cat([seqs[i][1][1][:lens[i]] for i in some]),
                    torch.cat([seqs[i][2][1][:lens[i]] for i in some]))
    total = [np.zeros((n_kv, n + steps)) for n in lens]
    for st in range(steps):
        row = lambda j: torch.stack([s[j][1][n + st] for s, n in zip(seqs, lens)])
        got = attn(c, 0, ids, None, [n + st for n in lens], row(0), row(1), row(2), True)
        for i, (s, n) in enumerate(zip(seqs, lens)):
            k, v = (c.held(s[j][0][:n + st + 1]) for j in (1, 2))
            ref, mag, w = kv8.attention(s[0][0][n + st:n + st + 1], k, v, n + st)
            c.close(got[i:i + 1], ref, mag)
            total[i][:, :n + st + 1] += w[0].reshape(n_kv, -1, n + st + 1).sum(1)
    ends = [n + steps for n in lens]
    buf = torch.full((n_kv * sum(ends),), -1.0, device="cuda")
    c.ctx.kv8_weights(c.desc, ss.SS_OUT, ids, buf)
    got, t = buf.double().cpu().numpy(), 0
    for n, ref in zip(ends, total):
        w = got[t:t + n_kv * n].reshape(n_kv, n)
        # the scores' error in the exponent (2^-15 at a score of 40), twice: of the token's own and of the sum
        np.testing.assert_allclose(w, ref, rtol=2.0 ** -12, atol=1e-12)
        t += n_kv * n


def test_a_step_may_be_repeated_and_the_cache_cut_back():
    rng = np.random.default_rng(10)
    c = Cache(wl.BF16, 4, 2, 128)
    q, k, v = c.tokens(rng, 64, 4), c.tokens(rng, 64, 2), c.tokens(rng, 64, 2)
    c.ctx.kv8_write(c.desc, 0, [0], [31], [0], k[1][:31], v[1][:31])
    step = lambda p, j: attn(c, 0, [0], None, [p], q[1][j:j + 1], k[1][j:j + 1], v[1][j:j + 1], True)
    a, b = step(31, 31), step(31, 31)                           # the block closes, twice
    assert np.array_equal(a, b)
    step(31, 40)                                                # another token in its place
    ref, mag, _ = kv8.attention(q[0][40:41], *(c.held(np.concatenate([x[0][:31], x[0][40:41]])) for x in (k, v)), 31)
    c.close(step(31, 40), ref, mag)
    c.ctx.kv8_write(c.desc, 0, [0], [20], [16], k[1][30:50], v[1][30:50])      # back to the second block
    assert c.ctx.kv_seq_len(c.desc, 0) == 36
    want = np.concatenate([k[0][:16], k[0][30:50]])
    c.same(c.export([0], [36])[0][0, 0], c.held(want))
    c.ctx.kv8_write(c.desc, 0, [0], [2], [0], k[1][5:7], v[1][5:7])            # back to nothing
    c.same(c.export([0], [2])[0][0, 1], c.held(v[0][5:7]))


def test_rows_of_a_fused_buffer_and_a_stream_of_their_own():
    rng = np.random.default_rng(11)
    c = Cache(wl.F16, 6, 2, 64)
    n = 50
    q, k, v = c.tokens(rng, n, 6), c.tokens(rng, n, 2), c.tokens(rng, n, 2)
    fused = torch.cat([q[1], k[1], v[1], torch.zeros_like(k[1])], dim=1)       # rows of 12 heads
    out = torch.empty(n, 6, 64, device="cuda", dtype=torch.float16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.ctx.kv8_attn_prefill(c.desc, 0, [0], [n], [0], fused[:, :6], fused[:, 6:8], fused[:, 8:10], out, s.cuda_stream)
    s.synchronize()
    ref, mag, _ = kv8.attention(q[0], c.held(k[0]), c.held(v[0]), 0)
    c.close(out.double().cpu().numpy(), ref, mag)


@pytest.mark.parametrize("dtype,n_kv,d", [(wl.BF16, 2, 128), (wl.F16, 1, 64), (wl.F32, 3, 64)])
def test_what_other_tokens_left_behind_is_not_seen(dtype, n_kv, d):
    """Pages and open blocks of freed sequences that held NaN, infinities and large values; and a NaN in a later block leaves earlier
    queries alone."""
    rng = np.random.default_rng(12)
    c = Cache(dtype, 2 * n_kv, n_kv, d, pages=24, seqs=2, weights=True)
    n = 16 * 11 + 9
    junk = torch.full((n, n_kv, d), float("nan"), device="cuda", dtype=TYPES[dtype])
    junk[::3] = float("inf")
    c.ctx.kv8_write(c.desc, 0, [5, 6], [n, n], [0, 0], torch.cat([junk, junk]), torch.cat([junk, junk]))
    c.ctx.kv_free(c.desc, [5, 6])
    lens = [1, 150]
    s = [[c.tokens(rng, m, 2 * n_kv), c.tokens(rng, m, n_kv), c.tokens(rng, m, n_kv)] for m in lens]
    got = attn(c, 0, [0, 1], lens, [0, 0], *(torch.cat([x[j][1] for x in s]) for j in range(3)), False)
    t = 0
    for x, m in zip(s, lens):
        ref, mag, _ = kv8.attention(x[0][0], c.held(x[1][0]), c.held(x[2][0]), 0)
        c.close(got[t:t + m], ref, mag)
        t += m
    more = [[c.tokens(rng, 1, 2 * n_kv), c.tokens(rng, 1, n_kv), c.tokens(rng, 1, n_kv)] for _ in lens]
    got = attn(c, 0, [0, 1], None, lens, *(torch.cat([x[j][1] for x in more]) for j in range(3)), True)
    for i, (x, y, m) in enumerate(zip(s, more, lens)):
        ref, mag, _ = kv8.attention(y[0][0], c.held(np.concatenate([x[1][0], y[1][0]])), c.held(np.concatenate([x[2][0], y[2][0]])), m)
        c.close(got[i:i + 1], ref, mag)
    # a NaN key in the last full block (positions 128 - 143) of sequence 1, a NaN value in its neighbour's
    k, v = s[1][1][1].clone(), s[1][2][1].clone()
    k[130] = float("nan")
    v[114] = float("nan")
    got = attn(c, 0, [1], [150], [0], s[1][0][1], k, v, False)
    ref, mag, _ = kv8.attention(s[1][0][0][:112], c.held(s[1][1][0][:112]), c.held(s[1][2][0][:112]), 0)
    c.close(got[:112], ref, mag)
    assert np.isnan(got[112:]).all()


@pytest.mark.parametrize("dtype,n_kv,d,layers", [(wl.BF16, 2, 128, 2), (wl.F16, 3, 64, 1), (wl.F32, 1, 128, 1)])
def test_eviction(dtype, n_kv, d, layers):
    rng = np.random.default_rng(13)
    c = Cache(dtype, 2 * n_kv, n_kv, d, layers=layers, pages=600, weights=True)
    lens = [1, 40, 64, 65, 130, 400, 1500, 90, 300]
    keep = [1, 1, 64, 64, 33, 256, 700, 200, 17]
    recent = 9
    ids = list(range(len(lens)))
    toks = [[(c.tokens(rng, n, n_kv), c.tokens(rng, n, n_kv)) for _ in range(layers)] for n in lens]
    w = [np.round(rng.exponential(size=(layers, n_kv, n)) * 8).astype(np.float32) / 8 for n in lens]      # many ties
    w[4][0, 0, 7] = np.nan
    w[4][0, 0, 90] = np.inf
    w[5][0, 0, :] = 0
    w[5][0, -1, ::2] = -0.0
    w[5][0, -1, 1::2] = 0
    w[6][0, 0, :300] *= -1
    c.ctx.kv_import_dev(c.desc, ids, lens, torch.cat([x[1].permute(1, 0, 2).reshape(-1) for s in toks for l in s for x in l]))
    c.ctx.kv8_weights(c.desc, ss.SS_IN, ids, torch.from_numpy(np.concatenate([x.reshape(-1) for x in w])).cuda())
    free = c.ctx.kv_free_pages(c.desc)
    c.ctx.kv8_evict(c.desc, ids, keep, recent)
    ends = [min(n, m) for n, m in zip(lens, keep)]
    assert [c.ctx.kv_seq_len(c.desc, i) for i in ids] == ends
    assert c.ctx.kv_free_pages(c.desc) - free == sum((n + 15) // 16 - (m + 15) // 16 for n, m in zip(lens, ends))
    store = lambda x: wl.round_to_storage(x, dtype)
    buf = torch.empty(layers * n_kv * sum(ends), device="cuda")
    c.ctx.kv8_weights(c.desc, ss.SS_OUT, ids, buf)
    got_w, t, refs = buf.cpu().numpy(), 0, []
    for i, got in enumerate(c.export(ids, ends)):
        for l in range(layers):
            k, v, kw = kv8.evict(*(kv8.units(x[0], dtype == wl.F32) for x in toks[i][l]), w[i][l], keep[i], recent, store, dtype == wl.F32)
            if l == 0:
                refs.append((k, v))
            c.same(got[l, 0], k)
            c.same(got[l, 1], v)
            np.testing.assert_array_equal(got_w[t:t + kw.size].reshape(kw.shape), kw)
            t += kw.size
    # decoding goes on: positions count on, the cache is what stayed
    q, k, v = (c.tokens(rng, len(ids), h) for h in (2 * n_kv, n_kv, n_kv))
    got = attn(c, 0, ids, None, lens, q[1], k[1], v[1], True)
    for i in ids:
        kk, vv = (np.concatenate([r, x[0][i:i + 1]]) for r, x in zip(refs[i], (k, v)))
        full = ends[i] // 16 * 16
        kk, vv = (np.concatenate([x[:full], c.held(x[full:])]) for x in (kk, vv))
        ref, mag, _ = kv8.attention(q[0][i:i + 1], kk, vv, ends[i])
        c.close(got[i:i + 1], ref, mag)


def _refused(code, fn, *a):
    with pytest.raises(ss.SeesawError) as e:
        fn(*a)
    assert e.value.code == code, e.value


def test_refusals():
    rng = np.random.default_rng(14)
    c = Cache(wl.BF16, 4, 2, 64, pages=8, seqs=3, max_len=100, layers=2)
    q, k, v = (c.tokens(rng, 100, h)[1] for h in (4, 2, 2))
    out = torch.empty_like(q)
    w = lambda ids, lens, at, n=None: c.ctx.kv8_write(c.desc, 0, ids, lens, at, k[:sum(lens)], v[:sum(lens)])
    other = ss.ShardDesc(ss.SS_TP, 2, 0, 0, 2)
    _refused(ss.SS_EINVAL, c.ctx.kv8_write, other, 0, [0], [4], [0], k[:4, :1], v[:4, :1])      # not in 8 bits
    _refused(ss.SS_EINVAL, c.ctx.kv8_enable, c.desc, 4)                                          # twice
    _refused(ss.SS_EINVAL, c.ctx.kv8_enable, other, 0)
    _refused(ss.SS_EINVAL, w, [0, 0], [2, 2], [0, 0])                                            # listed twice, unknown
    w([0], [40], [0])
    _refused(ss.SS_EINVAL, w, [0, 0], [2, 2], [40, 42])                                          # and known
    _refused(ss.SS_ENOENT, w, [0], [2], [41])
    _refused(ss.SS_EINVAL, w, [0], [2], [31])
    _refused(ss.SS_EINVAL, w, [0], [0], [40])
    _refused(ss.SS_EINVAL, w, [0], [61], [40])                                                   # beyond max_seq_len
    _refused(ss.SS_EINVAL, w, [0], [2], [-1])
    _refused(ss.SS_ENOENT, w, [9], [2], [16])
    _refused(ss.SS_EINVAL, c.ctx.kv8_write, c.desc, 2, [0], [2], [40], k[:2], v[:2])             # no such layer
    free = c.ctx.kv_free_pages(c.desc)
    _refused(ss.SS_ENOMEM, w, [1, 2], [60, 30], [0, 0])                                          # 3 + 4 + 2 of 8 pages
    _refused(ss.SS_ENOMEM, w, [1, 2, 3], [1, 1, 1], [0, 0, 0])                                   # four of three sequences
    assert c.ctx.kv_free_pages(c.desc) == free
    _refused(ss.SS_ENOENT, c.ctx.kv_seq_len, c.desc, 1)
    a = lambda at, n: c.ctx.kv8_attn_prefill(c.desc, 0, [0], [n], [at], q[:n], None, None, out[:n])
    _refused(ss.SS_ENOENT, a, 30, 11)
    a(30, 10)
    d = lambda at, kk, vv: c.ctx.kv8_attn_decode(c.desc, 0, [0], [at], q[:1], kk, vv, out[:1])
    _refused(ss.SS_EINVAL, d, 40, k[:1], None)
    _refused(ss.SS_ENOENT, d, 40, None, None)
    # rows: not aligned, too close together, of another type or number
    wide = torch.zeros(4, 2 * 64 + 4, device="cuda", dtype=torch.bfloat16)
    _refused(ss.SS_EINVAL, c.ctx.kv8_write, c.desc, 0, [0], [4], [40], wide[:, :128], v[:4])
    _refused(ss.SS_EINVAL, c.ctx.kv8_write, c.desc, 0, [0], [1], [40], wide[:1, 4:132], v[:1])
    _refused(ss.SS_EINVAL, c.ctx.kv8_write, c.desc, 0, [0], [4], [40], k[:1].expand(4, 2, 64), v[:4])
    for bad in (k[:4].float(), k[:3], k[:4].cpu(), k[:4].transpose(1, 2), q[:4]):
        with pytest.raises(ValueError):
            c.ctx.kv8_write(c.desc, 0, [0], [4], [40], bad, v[:4])
    with pytest.raises(ValueError):
        c.ctx.kv8_attn_decode(c.desc, 0, [0], [39], q[:1], None, None, out[:2])
    # layers that hold different numbers of tokens are not moved as a whole; no weights, no eviction
    buf = torch.empty(1 << 16, device="cuda", dtype=torch.bfloat16)
    _refused(ss.SS_EINVAL, c.ctx.kv_export_dev, c.desc, [0], buf)
    _refused(ss.SS_EINVAL, c.ctx.kv8_weights, c.desc, ss.SS_OUT, [0], torch.empty(1000, device="cuda"))
    _refused(ss.SS_EINVAL, c.ctx.kv8_evict, c.desc, [0], [3], 1)
    c.ctx.kv8_write(c.desc, 1, [0], [40], [0], k[:40], v[:40])
    c.ctx.kv_export_dev(c.desc, [0], buf)
    torch.cuda.synchronize()
    # a captured graph would hold the page lists of now
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        _refused(ss.SS_EHIP, lambda: c.ctx.kv8_attn_prefill(c.desc, 0, [0], [1], [39], q[:1], None, None, out[:1], s.cuda_stream))
        out.zero_()


def test_refusals_of_eviction():
    rng = np.random.default_rng(15)
    c = Cache(wl.F16, 2, 1, 64, weights=True)
    k, q = c.tokens(rng, 60, 1)[1], c.tokens(rng, 60, 2)[1]
    c.ctx.kv8_write(c.desc, 0, [0, 1], [50, 10], [0, 0], k, k)
    _refused(ss.SS_EINVAL, c.ctx.kv8_evict, c.desc, [0, 0], [20, 20], 4)
    _refused(ss.SS_EINVAL, c.ctx.kv8_evict, c.desc, [0], [0], 0)
    _refused(ss.SS_EINVAL, c.ctx.kv8_evict, c.desc, [0], [8], -1)
    _refused(ss.SS_ENOENT, c.ctx.kv8_evict, c.desc, [0, 7], [20, 20], 4)
    assert c.ctx.kv_seq_len(c.desc, 0) == 50
    c.ctx.kv8_evict(c.desc, [0, 1], [20, 20], 4)
    c.ctx.kv8_evict(c.desc, [], [], 4)
    assert (c.ctx.kv_seq_len(c.desc, 0), c.ctx.kv_seq_len(c.desc, 1)) == (20, 10)
    w = lambda at: c.ctx.kv8_write(c.desc, 0, [0], [3], [at], k[:3], k[:3])
    _refused(ss.SS_EINVAL, w, 49)                                # before the eviction
    _refused(ss.SS_EINVAL, w, 0)
    _refused(ss.SS_ENOENT, w, 51)
    w(50)
    w(50)
    assert c.ctx.kv_seq_len(c.desc, 0) == 23
    out = torch.empty(1, 2, 64, device="cuda", dtype=torch.float16)
    a = lambda at: c.ctx.kv8_attn_decode(c.desc, 0, [0], [at], q[:1], None, None, out)
    _refused(ss.SS_EINVAL, a, 48)
    a(49)                                                        # the newest token that stayed
    torch.cuda.synchronize()
