"""The offline loop over shards whose 8-bit caches have room for few sequences: prompts' shard, decode shard, both."""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import scheduler as sc

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2503_06433_amd as ss
    from paper_2503_06433_amd.harness import make_context, pp_desc, tp_desc


@pytest.mark.parametrize("prompt_seqs,decode_seqs", [(3, None), (None, 2), (3, 4), (1, 1), (64, 64)])
def test_loop_over_shards_with_room_for_few_sequences(prompt_seqs, decode_seqs):
    cfg = wl.config1().cfg
    raws = [wl.make_layer_weights(cfg, 500 + l)[1] for l in range(cfg.n_layers)]
    _, hr = wl.make_head_weights(cfg, 599)
    rng = np.random.default_rng(81)
    prompts = [rng.integers(0, cfg.vocab, size=int(n)).astype(np.int32) for n in rng.integers(2, 40, 13)]
    outs = [int(x) for x in rng.integers(1, 7, 13)]
    pages, tier_tokens, mpt, mds = 64, 120, 100, 6
    tok = 2 * cfg.n_kv_heads * cfg.head_dim * 4 * cfg.n_layers
    ctx = make_context(cfg, pages=pages, tier_bytes=tier_tokens * tok, pinned_bytes=1 << 20, max_seq_len=128)
    ctx.load_head(hr["embed"], hr["gf"], hr["wlm"])
    p, t = pp_desc(cfg), tp_desc(cfg, 1, 0)
    for d, seqs in ((p, prompt_seqs), (t, decode_seqs)):
        if seqs:
            ctx.kv8_enable(d, max_seqs=seqs)
        for l in range(cfg.n_layers):
            ctx.load_layer(d, l, raws[l])
    for _ in range(2):                                      # all room is there again behind a run
        toks, trace, stats = ctx.offline_run(p, t, prompts, outs, mpt, mds, reshard_weights=False)
        ref, ref_stats = sc.simulate([len(x) for x in prompts], outs, tier_tokens, pages, mpt, mds, cfg.page_size, 0, prompt_seqs, decode_seqs)
        assert trace == ref and stats["tokens"] == ref_stats["tokens"] == sum(outs)
        assert ctx.kv_free_pages(p) == pages and ctx.kv_free_pages(t) == pages
        assert [len(x) for x in toks] == outs
        for d, seqs in ((p, prompt_seqs), (t, decode_seqs)):
            if seqs:
                assert ctx.kv8_free_seqs(d) == seqs
            else:
                with pytest.raises(ss.SeesawError):
                    ctx.kv8_free_seqs(d)
    ctx.destroy()
