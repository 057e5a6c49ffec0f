"""Numbers next to half a step of their block, and evictions of values that are not finite: what the cache holds of them, exactly.

A block of the largest magnitude M (a whole number of at most 11 bits, M >= 2^10) holds v = m 2^-j as q = rint(127 v / M).  127 v / M is
(254 m - (2 k + 1) M 2^j) / (2 M 2^j) away from half a step k + 1 / 2: 0 or at least 1 / (2 M 2^j) > 2^-(12 + j).  It is below
127 * 2 * 2^-j < 2^(8 - j), and the fp32 quotient of the exact product 127 v is off by 2^-24 of that at most, 2^-(16 + j): on the right
side, or exactly on the half step.  For the types' widths the nearest two m of every (M, j, k) are gone through here."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from oracle import kv8
from test_gpu_kv8 import Cache, TYPES

torch = pytest.importorskip("torch")


def nearest(bits, big):
    """Values of `bits` significant bits, at most `big`, whose 127-fold quotient by big lies next to a half step: float64, exact."""
    lo, hi = 1 << (bits - 1), 1 << bits
    out = []
    for j in range(0, 9):
        k = np.arange(0, 127)
        m = (2 * k + 1) * big * 2 ** j // 254
        for c in (m, m + 1):
            c = c[(c >= lo) & (c < hi)]
            v = c * 2.0 ** -j
            out.append(v[v <= big])
    return np.unique(np.concatenate(out))


@pytest.mark.parametrize("bits", [8, 11])
def test_fp32_quotients_next_to_half_a_step_round_as_real_ones(bits):
    worst = np.inf
    for big in range(1 << (bits - 1), 1 << bits):
        v = nearest(bits, big)
        num = np.array([int(x) for x in v * 256 * 254], dtype=object)       # 254 v 2^8, whole numbers
        q, half = num // (2 * 256 * big), (num - 256 * big) % (2 * 256 * big) == 0
        up = num - q * (2 * 256 * big) > 256 * big
        even = half & (q % 2 == 1)
        want = (q + (up | even)).astype(np.int64)
        got = np.rint(v.astype(np.float32) * np.float32(127) / np.float32(big))
        assert np.array_equal(got, want), big
        t = v * 127 / big
        d = np.abs(t - np.floor(t) - 0.5)
        worst = min(worst, d[d > 0].min())
    assert worst < 2.0 ** (-18 if bits == 11 else -13)                      # they do come that near


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bits", [(wl.BF16, 8), (wl.F16, 11)])
def test_the_cache_rounds_them_so(dtype, bits):
    bigs = list(range(1 << (bits - 1), 1 << bits))
    x = np.zeros((16 * len(bigs), 1, 64))
    for i, big in enumerate(bigs):
        v = nearest(bits, big)
        assert 0 < len(v) < 1023
        v = np.concatenate([v, -v[:1023 - len(v)], [big]])
        b = np.zeros(1024)
        b[:len(v)] = v
        x[16 * i:16 * i + 16, 0] = b.reshape(16, 64)
    vals, raw = wl.quantize(x, dtype)
    assert np.array_equal(vals, x)
    t = torch.from_numpy(raw.view(np.int16)).cuda().view(TYPES[dtype])
    c = Cache(dtype, 1, 1, 64, pages=len(bigs), max_len=16 * len(bigs))
    c.ctx.kv8_write(c.desc, 0, [0], [len(x)], [0], t, t.flip(0).contiguous())
    k, v = c.export([0], [len(x)])[0][0]
    a = np.repeat(bigs, 16)[:, None, None]
    # one step is 1 / 127 of the largest: the exported value, rounded to 8 or 11 bits, still names its whole number
    assert np.array_equal(np.rint(k * 127 / a), np.rint(kv8.held(x) * 127 / a))
    assert np.array_equal(np.rint(v * 127 / a[::-1]), np.rint(kv8.held(x[::-1]) * 127 / a[::-1]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(wl.BF16, 128), (wl.F16, 64), (wl.F32, 64)])
def test_infinite_values_that_stay_in_the_open_block_come_back(dtype, d):
    """Evictions whose newest tokens, infinities and NaN among them, end in the open block: each as it was; those that end in a full block
    make that block NaN."""
    rng = np.random.default_rng(51)
    c = Cache(dtype, 2, 2, d, pages=64, weights=True)
    lens, keep = [45, 90, 60], [9, 40, 33]
    toks = []
    for n in lens:
        pair = []
        for part in range(2):
            x, _ = wl.quantize(rng.normal(size=(n, 2, d)), dtype)
            x[n - 1, 0, 3 + part], x[n - 2, 1, 5], x[n - 3, part, 7] = np.inf, -np.inf, np.nan
            x[n - 4, 0, :] = -np.inf
            if n == 60:
                x[n - 20, 1, 2] = np.inf                     # in the cut cache's second full block
            _, raw = wl.quantize(np.where(np.isnan(x), 0, x), dtype)
            t = torch.from_numpy(raw if dtype == wl.F32 else raw.view(np.int16)).cuda()
            t = (t if dtype == wl.F32 else t.view(TYPES[dtype])).clone()
            t[torch.from_numpy(np.isnan(x)).cuda()] = float("nan")
            pair.append((x, t))
        toks.append(pair)
    w = [np.concatenate([rng.exponential(size=(2, n - 24)), np.full((2, 24), 50.0)], axis=1).astype(np.float32) for n in lens]
    ids = [0, 1, 2]
    c.ctx.kv_import_dev(c.desc, ids, lens, torch.cat([x[1].permute(1, 0, 2).reshape(-1) for s in toks for x in s]))
    c.ctx.kv8_weights(c.desc, ss.SS_IN, ids, torch.from_numpy(np.concatenate([x.reshape(-1) for x in w])).cuda())
    c.ctx.kv8_evict(c.desc, ids, keep, 8)
    infinite = 0
    for i, got in enumerate(c.export(ids, keep)):
        ref = kv8.evict(*(kv8.units(x[0], dtype == wl.F32) for x in toks[i]), w[i], keep[i], 8, lambda a: wl.round_to_storage(a, dtype), dtype == wl.F32)
        for part in range(2):
            r, g = ref[part], got[0, part]
            open_ = keep[i] // 16 * 16
            assert np.array_equal(np.isnan(g), np.isnan(r)) and np.array_equal(g[np.isinf(r)], r[np.isinf(r)])
            assert np.array_equal(np.isinf(g), np.isinf(r))
            infinite += int(np.isinf(r[open_:]).sum())
            fin = np.isfinite(r)
            c.same(g[fin], r[fin])
    assert infinite == 2 * (2 * (d + 2) + 1)                 # the first two sequences' all, of the third's the newest token's
