"""Attention of 16-bit models over 8-bit caches whose values differ widely in size: open blocks of half values, caches of the smallest and
of the largest brain-float values, blocks of zeros beside large ones.

Tolerance: that of test_gpu_kv8 (a half step H of the type for the output, H for the rounded weights and 2^-11 for the scores, both times the
sum of the weights times |v|), without its absolute term: below the type's normal range numbers are 2^-133 apart (brain float) or
2^-24 (half), half of that is the rounding of the output."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from oracle import kv8
from test_gpu_kv8 import H, SLACK, TYPES, Cache, attn

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LAST = {wl.BF16: 2.0 ** -134, wl.F16: 2.0 ** -25}


def _dev(raw, dtype):
    return torch.from_numpy(raw.view(np.int16)).cuda().view(TYPES[dtype])


def _close(got, ref, mag, dtype):
    assert got.shape == ref.shape and np.isfinite(got).all()
    bound = (H[dtype] * (np.abs(ref) + mag) + SLACK[dtype] * mag) * (1 + 2.0 ** -10) + LAST[dtype] * (1 + 2.0 ** -10)
    worst = np.max(np.abs(got - ref) / bound)
    assert worst <= 1, "off by %.2f of the bound" % worst


def _both(c, q, k, v, n_last=3):
    """Prompt of the whole sequence, then its last tokens as steps of another one: outputs against the statement.  q, k, v: pairs of float64
    and device tensors."""
    n = k[0].shape[0]
    hk, hv = c.held(k[0]), c.held(v[0])
    got = attn(c, 0, [1], [n], [0], q[1], k[1], v[1], False)
    ref, mag, _ = kv8.attention(q[0], hk, hv, 0)
    _close(got, ref, mag, c.dtype)
    m = n - n_last
    c.ctx.kv8_write(c.desc, 0, [2], [m], [0], k[1][:m], v[1][:m])
    w = np.zeros((c.n_kv, n))
    for p in range(m, n):
        got = attn(c, 0, [2], None, [p], q[1][p:p + 1], k[1][p:p + 1], v[1][p:p + 1], True)
        kk, vv = c.held(k[0][:p + 1]), c.held(v[0][:p + 1])
        ref, mag, wt = kv8.attention(q[0][p:p + 1], kk, vv, p)
        _close(got, ref, mag, c.dtype)
        w[:, :p + 1] += wt[0].reshape(c.n_kv, -1, p + 1).sum(1)
    buf = torch.full((c.n_kv * n,), -1.0, device="cuda")
    c.ctx.kv8_weights(c.desc, ss.SS_OUT, [2], buf)
    np.testing.assert_allclose(buf.double().cpu().numpy().reshape(c.n_kv, n), w, rtol=2.0 ** -12, atol=1e-12)
    c.ctx.kv_free(c.desc, [1, 2])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("big", [65504.0, 60000.0, 300.0, 128.0, 127.0, 2.0 ** -10])
def test_small_values_next_to_large_ones_in_an_open_block_of_halves(big, d):
    """All weight (64 nats) on a token whose values are some 2^-24 of its neighbour's."""
    rng = np.random.default_rng(41)
    c = Cache(wl.F16, 4, 2, d, weights=True)
    for n in (9, 27):
        qv, kv_, vv = rng.normal(size=(n, 4, d)), rng.normal(size=(n, 2, d)) * 0.1, rng.normal(size=(n, 2, d))
        heavy = n - 5
        vv[heavy] = rng.uniform(-1, 1, size=(2, d)) * big * 2.0 ** -24 + np.sign(rng.normal(size=(2, d))) * big * 2.0 ** -25
        vv[n - 6], vv[n - 7, 0] = big, -big
        kv_[:, :, 0] = 0
        kv_[heavy, :, 0] = 2 * np.sqrt(d)
        qv[:, :, 0] = 32
        q, k, v = ((x, _dev(r, wl.F16)) for x, r in (wl.quantize(a, wl.F16) for a in (qv, kv_, vv)))
        _both(c, q, k, v)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [-118, -112, -100, -60, 60, 100, 120])
def test_caches_of_small_and_of_large_values(scale, d):
    """All values of a cache around 2^scale."""
    rng = np.random.default_rng(42)
    c = Cache(wl.BF16, 6, 2, d, pages=300, weights=True)
    for n in (5, 47, 1100):
        v, r = wl.quantize(np.clip(rng.normal(size=(n, 2, d)), -3, 3) * 2.0 ** scale, wl.BF16)
        _both(c, c.tokens(rng, n, 6), c.tokens(rng, n, 2), (v, _dev(r, wl.BF16)))


# powers of two of a cycle of blocks; None: zeros
CYCLES = [(None, 110), (110, None), (None, None, None, None, None, 115, None), (0, 110), (110, 0, -60), (-100, None, 0, 100, -30),
          (-110, 0), (0, -110, -110, -110, -110), (None, -110),
          (0,) * 40 + (110,) + (None,) * 20 + (0,) * 30]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cycle", CYCLES, ids=["_".join("zero" if x is None else str(x) for x in c[:8]) for c in CYCLES])
def test_blocks_of_very_different_size_side_by_side(cycle, d):
    """Weights of similar size on blocks of zeros, of ordinary, tiny and huge values: what a block does not add to the output it still adds
    to the sum of weights."""
    rng = np.random.default_rng(43)
    c = Cache(wl.BF16, 3, 1, d, pages=500, weights=True)
    for n in (13, 16 * len(cycle) + 7, 700, 2500):
        x = np.clip(rng.normal(size=(n, 1, d)), -3, 3)
        for b in range(0, n, 16):
            e = cycle[b // 16 % len(cycle)]
            x[b:b + 16] *= 0.0 if e is None else 2.0 ** e
        v, r = wl.quantize(x, wl.BF16)
        _both(c, c.tokens(rng, n, 3, 0.5), c.tokens(rng, n, 1, 0.5), (v, _dev(r, wl.BF16)))
