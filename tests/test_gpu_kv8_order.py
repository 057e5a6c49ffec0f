"""Attention right behind a swap-in, without a wait of the caller's: calls over an 8-bit cache wait for queued movements of their
sequences, those that write nothing as well."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from oracle import kv8
from test_gpu_kv8 import H, SLACK

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [wl.BF16, wl.F32])
def test_attention_right_behind_a_swap_in(dtype):
    from paper_2503_06433_amd import harness as hz
    n_q, n_kv, d, layers = 4, 2, 128, 3
    lens, ids = [2000, 37, 1500, 160], [4, 1, 9, 6]
    ctx = ss.Context(ss.ModelCfg(n_q * d, n_q, n_kv, d, 64, layers, 0, 1e-5, 10000.0, dtype, 16), ss.RuntimeCfg(400, 64 << 20, 16 << 20, 0, 4096))
    src, dst = ss.ShardDesc(ss.SS_PP, 1, 0, 0, layers), ss.ShardDesc(ss.SS_TP, 1, 0, 0, layers)
    ctx.kv8_enable(dst, 8, True)
    rng = np.random.default_rng(71)
    vals, raw = zip(*[wl.quantize(rng.normal(size=(layers, 2, n_kv, n, d)), dtype) for n in lens])
    ctx.kv_import_dev(src, ids, lens, hz.to_device(np.concatenate([r.reshape(-1) for r in raw]), dtype))
    ctx.kv_swap(src, ss.SS_OUT, ids)
    ctx.sync()
    qv, qr = wl.quantize(rng.normal(size=(4 * 5, n_q, d)), dtype)
    q = hz.to_device(qr.reshape(-1), dtype).view(-1, n_q, d)
    torch.cuda.synchronize()
    for turn in range(4):
        ctx.kv_swap(dst, ss.SS_IN, ids)
        layer = turn % layers
        if turn % 2:
            out = torch.empty(20, n_q, d, device="cuda", dtype=q.dtype)
            ctx.kv8_attn_prefill(dst, layer, ids, [5] * 4, [n - 5 for n in lens], q, None, None, out)
            rows = 5
        else:
            out = torch.empty(4, n_q, d, device="cuda", dtype=q.dtype)
            ctx.kv8_attn_decode(dst, layer, ids, [n - 1 for n in lens], q[:4], None, None, out)
            rows = 1
        torch.cuda.synchronize()
        got = out.double().cpu().numpy()
        for i, (x, n) in enumerate(zip(vals, lens)):
            k, v = (kv8.held(x[layer, p].transpose(1, 0, 2)) for p in range(2))
            ref, mag, _ = kv8.attention(qv[i * rows:(i + 1) * rows], k, v, n - rows)
            err = np.abs(got[i * rows:(i + 1) * rows] - ref)
            assert np.all(err <= H[dtype] * (np.abs(ref) + mag) + SLACK[dtype] * mag), (turn, i)
        if not turn % 2:                                    # the weights are those of this step alone
            w = torch.empty(layers * n_kv * sum(lens), device="cuda")
            ctx.kv8_weights(dst, ss.SS_OUT, ids, w)
            assert abs(w.double().sum().item() - 4 * n_q) < 1e-3
        ctx.kv_free(dst, ids)
    ctx.destroy()
