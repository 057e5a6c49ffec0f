"""Decode steps of whole layer calls over an 8-bit cache, through blocks that open, fill and are quantised, against the oracle and against
what the cache is to hold of them.

Tolerance of the cache: keys and values come out of products whose inputs are rounded (bf16: 2^-9 of each of 512 terms, together 0.003 of the
values' rms, 0.013 for the worst of some ten thousand, which is 0.0045 of a block's largest, about three times the rms) and are rounded three times
more, as products, rotated and read back (2^-9 of the largest each, 0.006): 1.2e-2 of the block's largest; an eighth of it in half (1.5e-3); in
fp32 (sums of 512 products of 2^-24 each, not yet 2^-20 of the largest together: 1e-5).  A full block's are a half step of its largest from that, of
a largest that is off by as much."""
import numpy as np
import pytest

import torch

import workloads as wl
from oracle import kv8
from test_gpu_kv8_layer import _cfg, _close

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2503_06433_amd as ss
    from paper_2503_06433_amd import harness as hz
    from paper_2503_06433_amd.harness import make_context, pp_desc, to_device

TOL = {wl.F32: 1e-5, wl.BF16: 1.2e-2, wl.F16: 1.5e-3}


@pytest.mark.parametrize("dtype,d,n_q,n_kv", [(wl.BF16, 128, 20, 4), (wl.F16, 64, 18, 2), (wl.F32, 128, 6, 3), (wl.F32, 64, 3, 1), (wl.F16, 128, 9, 9)])
def test_steps_through_blocks(dtype, d, n_q, n_kv):
    cfg = _cfg(dtype, d, n_q, n_kv)
    vals, raws = wl.make_layer_weights(cfg, 15)
    ctx = make_context(cfg, pages=64)
    t = pp_desc(cfg)
    ctx.kv8_enable(t, max_seqs=6, weights=True)
    ctx.load_layer(t, 0, raws)
    cache = kv8.LayerCache()
    rk = lambda a: wl.round_to_storage(a, dtype)
    ids, lens = [3, 0, 8, 5], [14, 31, 1, 15]
    xv, xr = wl.make_activations((sum(lens), cfg.hidden), 16, dtype)
    out = hz.empty_like_acts(sum(lens), cfg.hidden, dtype)
    ctx.layer_prefill(t, 0, ss.SS_ATTN | ss.SS_NO_RESIDUAL, ids, lens, [0] * 4, to_device(xr, dtype), out)
    kv8.attn_block(cfg, vals, xv, [(i, n, 0) for i, n in zip(ids, lens)], cache, 1, 0, rk)
    for step in range(19):
        live = [j for j in range(4) if j != step % 4]                # not all of them every time
        xv, xr = wl.make_activations((3, cfg.hidden), 40 + step, dtype)
        out = hz.empty_like_acts(3, cfg.hidden, dtype)
        at = [lens[j] for j in live]
        ctx.layer_decode(t, 0, ss.SS_ATTN | ss.SS_NO_RESIDUAL, [ids[j] for j in live], at, to_device(xr, dtype), out)
        torch.cuda.synchronize()
        ref = kv8.attn_block(cfg, vals, xv, [(ids[j], 1, n) for j, n in zip(live, at)], cache, 1, 0, rk)
        _close(hz.to_f64(out, dtype), ref, dtype)
        for j in live:
            lens[j] += 1
    for i, n in zip(ids, lens):
        raw = ctx.kv_read(t, i, 0, n_kv)
        for x, y in zip(wl.storage_to_f64(raw, dtype), cache.data[i]):
            x = x.transpose(1, 0, 2)
            assert x.shape == y.shape == (n, n_kv, d)
            for b in range(0, n, 16):
                top = np.abs(y[b:b + 16]).max(axis=(0, 2), keepdims=True)
                half = (1 + TOL[dtype]) / 254 if b + 16 <= n else 0
                assert np.all(np.abs(x[b:b + 16] - y[b:b + 16]) <= (half + TOL[dtype]) * top), (i, b)
    ctx.destroy()
