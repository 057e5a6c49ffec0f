"""What is timed of the 8-bit KV cache: writing it, attention of single tokens and of prompts over it, eviction from it.

A block is 16 consecutive tokens of one kv head, K and V apart.  A full block holds whole numbers q = v * 127 / A, rounded to
the nearest (halves to even), of its largest magnitude A, and stands for q * (A / 127).  The last block of a sequence, while it
has fewer than 16 tokens, is kept in the model's type.

A case names the heads, the type and the lengths; the lengths belong to the case (`lens_seed`), so that its work is a fixed
number, everything else is drawn from the seed."""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 16
CHUNK_BYTES = 2 << 30          # of the largest temporary of a plain pass


def _case(op, dtype, n_q, n_kv, d, seqs, new, old=(0, 0), lens_seed=1, layers=1, weights=False, keep=0, recent=0, name=None):
    c = {"op": op, "dtype": dtype, "n_q": n_q, "n_kv": n_kv, "d": d, "seqs": seqs, "new_lo": new[0], "new_hi": new[1],
         "old_lo": old[0], "old_hi": old[1], "lens_seed": lens_seed, "layers": layers, "weights": weights, "keep": keep, "recent": recent}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one more token for each of 64 short chats of the tiny whole-model shape, blocks open and closing
        _case("write", "f32", 4, 4, 64, 64, (1, 1), (20, 60), 11, name="write_tokens_tiny_f32"),
        # four prompts of the 7B shape into the cache and out to staging, as for a swap
        _case("write", "bf16", 32, 32, 128, 4, (90, 310), lens_seed=12, name="write_prompts_7b"),
        # the prompts of a prefill batch of the 70B shape
        _case("write", "f16", 64, 8, 128, 32, (512, 4096), lens_seed=13, name="write_prompts_70b_f16"),
        # one user, one token, 7B shape: latency
        _case("decode", "bf16", 32, 32, 128, 1, (0, 0), (700, 700), 21, name="decode_7b_one_user"),
        # an offline batch of the 7B shape
        _case("decode", "bf16", 32, 32, 128, 256, (0, 0), (512, 2560), 22, name="decode_7b_b256"),
        # a shard of eight of the 70B shape: one kv head, a thousand sequences
        _case("decode", "f16", 8, 1, 128, 1024, (0, 0), (512, 4096), 23, name="decode_70b_tp8_b1024_f16"),
        # few sequences with long caches, the accumulated weights kept for eviction
        _case("decode", "bf16", 64, 8, 128, 6, (0, 0), (9000, 40000), 24, weights=True, name="decode_70b_long_weights"),
        # short prompts of odd lengths
        _case("prefill", "bf16", 10, 10, 128, 5, (1, 70), lens_seed=31, name="prefill_13b_tp4_short"),
        # chunks of four long prompts behind what is cached of them
        _case("prefill", "f16", 32, 32, 128, 4, (500, 520), (1000, 6000), 32, name="prefill_7b_chunks_f16"),
        # a prefill batch of the 70B shape
        _case("prefill", "bf16", 64, 8, 128, 24, (512, 4096), lens_seed=33, name="prefill_70b_b24"),
        # short chats over their budget, heads of 64
        _case("evict", "f16", 4, 4, 64, 16, (150, 700), lens_seed=41, keep=128, recent=32, name="evict_tiny_f16"),
        # long sequences of two layers of the 70B shape cut to 2048 tokens
        _case("evict", "bf16", 64, 8, 128, 16, (1500, 9000), lens_seed=42, layers=2, keep=2048, recent=256, name="evict_70b_long"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: the head layouts of the framework's shapes and generic ones, sizes over their
    logarithm; what would cost more than the largest listed case gets fewer sequences."""
    op = rng.choices(["decode", "prefill", "write", "evict"], [4, 3, 2, 2])[0]
    n_q, n_kv, d = rng.choice([(32, 32, 128), (10, 10, 128), (40, 40, 128), (64, 8, 128), (8, 1, 128), (32, 4, 128), (28, 4, 128),
                               (16, 1, 128), (4, 4, 64), (14, 2, 64), (32, 8, 64)])
    dtype = rng.choices(["bf16", "f16"], [2, 1])[0]
    seed = rng.randrange(1 << 20)
    if op == "decode":
        hi = _log_int(rng, 1, 32000)
        lo = max(1, int(hi * rng.choice([0.1, 0.5, 1.0])))
        room = max(1, int(5e8 / (2 * n_kv * d * (lo + hi) / 2)))
        return _case(op, dtype, n_q, n_kv, d, min(_log_int(rng, 1, 1024), room), (0, 0), (lo, hi), seed, weights=rng.random() < 0.3)
    if op == "prefill":
        hi = _log_int(rng, 2, 4096)
        old = rng.choice([0, 0, _log_int(rng, 16, 8000)])
        room = max(1, int(8e11 / (4 * n_q * d * hi * (old + hi))))
        return _case(op, dtype, n_q, n_kv, d, min(_log_int(rng, 1, 32), room), (max(1, hi // 3), hi), (old // 2, old), seed)
    if op == "write":
        one = rng.random() < 0.3
        hi = 1 if one else _log_int(rng, 2, 4096)
        old = _log_int(rng, 16, 500) if one else rng.choice([0, 0, _log_int(rng, 16, 2000)])
        room = max(1, int(7e7 / (n_kv * d * (hi + old))))
        return _case(op, dtype, n_q, n_kv, d, min(_log_int(rng, 1, 256), room), (max(1, hi // 4), hi), (old // 2, old), seed)
    hi = _log_int(rng, 40, 12000)
    keep = max(2, int(hi * rng.uniform(0.1, 0.9)))
    layers = rng.choice([1, 1, 2])
    room = max(1, int(1.4e8 / (n_kv * d * hi * layers)))
    return _case(op, dtype, n_q, n_kv, d, min(_log_int(rng, 1, 64), room), (max(1, hi // 4), hi), lens_seed=seed, layers=layers,
                 keep=keep, recent=int(keep * rng.choice([0.0, 0.1, 0.5])))


def _lens(case):
    """New and cached tokens of every sequence.  Chunks of several tokens begin at a block, as chunked prefill has them."""
    rng = random.Random(case["lens_seed"])
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    old = [rng.randint(case["old_lo"], case["old_hi"]) for _ in range(case["seqs"])]
    if case["new_hi"] > 1:
        old = [o // BLOCK * BLOCK for o in old]
    return new, old


def work(case):
    new, old = _lens(case)
    es = DTYPES[case["dtype"]].itemsize
    h, d, n_q = case["n_kv"], case["d"], case["n_q"]
    per_tok = 2 * h * d                                    # elements of K and V of a token
    held = lambda n: n // BLOCK * (BLOCK * per_tok + 8 * h) + n % BLOCK * per_tok * es      # bytes of a cache of n tokens
    if case["op"] == "decode":
        b = sum(held(o) for o in old) + 2 * case["seqs"] * n_q * d * es
        if case["weights"]:
            b += 2 * 4 * h * sum(old)                      # read, added to, written
        return {"bytes": b, "flops": 4 * n_q * d * sum(old)}
    if case["op"] == "evict":
        b = f = 0
        for n in new:
            kept = min(n, case["keep"])
            b += n * per_tok * es + kept * per_tok * es + held(n) + held(kept) + 4 * h * (n + kept)
            f += 4 * n * per_tok
        return {"bytes": b * case["layers"], "flops": f * case["layers"]}
    b = f = 0
    for n, o in zip(new, old):
        b += n * per_tok * es + held(o) + (held(o + n) - held(o // BLOCK * BLOCK)) + (o + n) * per_tok * es
        f += 4 * n * per_tok
        if case["op"] == "prefill":
            b += 2 * n * n_q * d * es
            f += 4 * n_q * d * (n * o + n * (n + 1) // 2)
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------------------------------------- inputs
def _inputs(case, seed):
    """Everything random of a case: queries, and keys and values of cached and new tokens, [tokens, heads, d] with the sequences
    back to back.  Keys have a few channels of several times the others' size, as rotated keys do; tokens differ in size."""
    new, old = _lens(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, h, d = DTYPES[case["dtype"]], case["n_kv"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def keys(n):
        channel = 1.0 + 3.0 * (torch.rand(h, d, generator=g, device="cuda") < 0.05)
        return (normal(n, h, d) * channel * torch.exp(0.2 * normal(n, 1, 1))).to(dt)

    def values(n):
        return (normal(n, h, d) * torch.exp(0.5 * normal(n, h, 1))).to(dt)

    x = {"new": new, "old": old}
    layers = case["layers"]
    if case["op"] == "evict":
        # what attention leaves behind: most weights small, a few large, some tokens never looked at (ties)
        for name, make in (("k", keys), ("v", values)):
            x[name] = [make(sum(new)) for _ in range(layers)]
        w = torch.exp(2.0 * normal(layers, h, sum(new)))
        x["w"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.1, torch.zeros_like(w), w)
        return x
    x["k_old"], x["v_old"] = keys(sum(old)), values(sum(old))
    if case["op"] != "decode":
        x["k"], x["v"] = keys(sum(new)), values(sum(new))
    n_queries = case["seqs"] if case["op"] == "decode" else sum(new)
    if case["op"] != "write":
        x["q"] = normal(n_queries, case["n_q"], d).to(dt)
    if case["weights"]:
        x["w"] = torch.rand(h * sum(old), generator=g, device="cuda") * 4.0
    return x


def _staging(lens, ks, vs):
    """[sequence][layer][K | V][head][position][d] of keys and values [tokens, heads, d] of every layer, flat."""
    out, t = [], 0
    for n in lens:
        for k, v in zip(ks, vs):
            out += [k[t:t + n].permute(1, 0, 2).reshape(-1), v[t:t + n].permute(1, 0, 2).reshape(-1)]
        t += n
    return torch.cat(out) if out else None


# ---------------------------------------------------------------------------------------------------- the plain form
class _Grid:
    """Tokens of sequences laid into blocks of 16: where each goes, and which blocks are full."""

    def __init__(self, begins, ends):
        at, full, first, blocks, tok = [], [], [], 0, 0
        for b, e in zip(begins, ends):
            b0 = b // BLOCK * BLOCK
            at.append(torch.arange(b, e) - b0 + blocks * BLOCK)
            first.append(blocks)
            n = (e + BLOCK - 1) // BLOCK - b0 // BLOCK
            full += [b0 + (i + 1) * BLOCK <= e for i in range(n)]
            blocks += n
        self.n = blocks
        self.at = torch.cat(at).cuda()
        self.full = torch.tensor(full, dtype=torch.bool, device="cuda")
        self.first = first


def _quantise(x, dtype=None):
    """Blocks [n, 16, h, d] in fp32 -> whole numbers and the largest magnitude [n, 1, h, 1].  The quotient of 16-bit numbers is never
    so close to half a step that 32 bits would round it the other way; that of 32-bit numbers is formed in 64."""
    a = x.abs().amax(dim=(1, 3), keepdim=True)
    div = torch.where(a > 0, a, torch.ones_like(a))
    if dtype is torch.float32:
        return torch.round(x.double() * 127.0 / div.double()).float(), a
    return torch.round(x * 127.0 / div), a


def _fill(x, grid):
    blocks = torch.zeros((grid.n * BLOCK,) + x.shape[1:], device="cuda", dtype=torch.float32)
    blocks[grid.at] = x.float()
    return blocks.view((grid.n, BLOCK) + x.shape[1:])


def _store(x, grid):
    """Tokens -> their blocks as the cache holds them: int8 numbers, magnitudes, and the tokens themselves (open blocks)."""
    b = _fill(x, grid)
    q, a = _quantise(b, x.dtype)
    return q.to(torch.int8), a, b.to(x.dtype)


def _held(q, a, open_, full):
    """What blocks stand for, fp32."""
    return torch.where(full.view(-1, 1, 1, 1), q.float() * (a / 127.0), open_.float())


def _rows(lens, h):
    """Rows (of K tokens x heads, then V tokens x heads) in the order of the staging layout."""
    rows, t, total = [], 0, sum(lens)
    for n in lens:
        for c in range(2):
            i = torch.arange(n).view(1, n) + t + c * total
            rows.append((i * h + torch.arange(h).view(h, 1)).reshape(-1))
        t += n
    return torch.cat(rows).cuda()


def _prepare_plain(case, x):
    s = dict(x)
    h, new, old = case["n_kv"], x["new"], x["old"]
    if case["op"] == "evict":
        s["staging"] = _staging(new, x["k"], x["v"])
        t, parts = 0, []
        for n in new:
            parts.append(x["w"][:, :, t:t + n].reshape(-1))
            t += n
        s["weights"] = torch.cat(parts)
        for name in ("k", "v", "w"):
            del s[name]
        return s
    if sum(old):
        grid = _Grid([0] * len(old), old)
        s["cache"] = _store(x["k_old"], grid), _store(x["v_old"], grid)
        s["cache_grid"] = grid
    del s["k_old"], s["v_old"]
    if case["op"] == "decode":
        # sequences of similar length together, so that little of a group is padding
        order = sorted(range(len(old)), key=lambda i: -old[i])
        groups, i = [], 0
        while i < len(order):
            blocks = (old[order[i]] + BLOCK - 1) // BLOCK
            n = max(1, CHUNK_BYTES // (blocks * BLOCK * h * case["d"] * 8))
            ids = order[i:i + n]
            table = torch.zeros(len(ids), blocks, dtype=torch.long)
            there = torch.zeros(len(ids), blocks * BLOCK, dtype=torch.bool)
            for j, sq in enumerate(ids):
                nb = (old[sq] + BLOCK - 1) // BLOCK
                table[j, :nb] = torch.arange(nb) + s["cache_grid"].first[sq]
                there[j, :old[sq]] = True
            groups.append((torch.tensor(ids).cuda(), table.cuda(), there.cuda()))
            i += n
        s["groups"] = groups
        if case["weights"]:
            # where the weight of (sequence, head, token) of a group lies in [sequence][head][token]
            base, o = [], 0
            for n in old:
                base.append(o)
                o += h * n
            s["w_at"] = []
            for ids, _, there in groups:
                j, p = torch.nonzero(there.cpu(), as_tuple=True)
                b = torch.tensor(base)[ids.cpu()][j]
                n = torch.tensor(old)[ids.cpu()][j]
                s["w_at"].append((b + p + torch.arange(h).view(h, 1) * n).cuda())
        return s
    s["grid"] = _Grid(old, [o + n for o, n in zip(old, new)])
    lens = [o + n for o, n in zip(old, new)]
    s["rows"] = _rows(lens, h)
    # every token of the sequences after the write: of a cached block, or of a written one
    src, written0 = [], s["cache_grid"].n * BLOCK if sum(old) else 0
    for i, (n, o) in enumerate(zip(new, old)):
        kept = o // BLOCK * BLOCK
        if kept:
            src.append(torch.arange(kept) + s["cache_grid"].first[i] * BLOCK)
        src.append(torch.arange(o + n - kept) + written0 + s["grid"].first[i] * BLOCK)
    s["tokens"] = torch.cat(src).cuda()
    # the cached tokens of a block that is open before the write
    frm, to = [], []
    for i, o in enumerate(old):
        if o % BLOCK:
            frm.append(torch.arange(o % BLOCK) + (s["cache_grid"].first[i] + o // BLOCK) * BLOCK)
            to.append(torch.arange(o % BLOCK) + s["grid"].first[i] * BLOCK)
    s["reopen"] = (torch.cat(frm).cuda(), torch.cat(to).cuda()) if frm else None
    return s


def _plain_write(case, s):
    """Keys and values [tokens, heads, d], fp32, that the cache stands for after the new tokens came."""
    grid, out = s["grid"], []
    for c, name in enumerate(("k", "v")):
        b = _fill(s[name], grid)
        if s["reopen"]:
            frm, to = s["reopen"]
            b.view((-1,) + b.shape[2:])[to] = s["cache"][c][2].view((-1,) + b.shape[2:])[frm].float()
        q, a = _quantise(b, s[name].dtype)
        blocks = _held(q, a, b, grid.full)
        if "cache" in s:
            blocks = torch.cat([_held(*s["cache"][c], s["cache_grid"].full), blocks])
        out.append(blocks.view((-1,) + blocks.shape[2:])[s["tokens"]])
    return out


def _softmax_parts(scores):
    p = torch.exp(scores - scores.amax(dim=-1, keepdim=True))
    return p, p.sum(dim=-1, keepdim=True)


def _plain_export(case, s, k, v):
    return torch.stack([k, v]).view(-1, case["d"])[s["rows"]].reshape(-1).to(DTYPES[case["dtype"]])


def _plain_prefill(case, s):
    k, v = _plain_write(case, s)
    h, d, n_q, dt = case["n_kv"], case["d"], case["n_q"], DTYPES[case["dtype"]]
    per = n_q // h
    out = torch.empty(sum(s["new"]), n_q, d, device="cuda", dtype=dt)
    t = qt = 0
    for n, o in zip(s["new"], s["old"]):
        ln = o + n
        step = max(1, CHUNK_BYTES // (4 * per * n * ln))
        seen = torch.arange(ln, device="cuda").view(1, 1, ln) <= torch.arange(o, ln, device="cuda").view(1, n, 1)
        for g in range(0, h, step):
            m = min(step, h - g)
            q = s["q"][qt:qt + n, g * per:(g + m) * per].float().view(n, m, per, d).permute(1, 2, 0, 3).reshape(m, per * n, d)
            kt = k[t:t + ln, g:g + m].permute(1, 2, 0).contiguous()
            sc = torch.bmm(q, kt).view(m * per, n, ln) / math.sqrt(d)
            p, l = _softmax_parts(sc.masked_fill_(~seen, float("-inf")))
            a = torch.bmm(p.view(m, per * n, ln), v[t:t + ln, g:g + m].permute(1, 0, 2).contiguous()) / l.view(m, per * n, 1)
            out[qt:qt + n, g * per:(g + m) * per] = a.view(m * per, n, d).permute(1, 0, 2).to(dt)
        t += ln
        qt += n
    return out, _plain_export(case, s, k, v)


def _plain_decode(case, s):
    h, d, n_q, dt = case["n_kv"], case["d"], case["n_q"], DTYPES[case["dtype"]]
    out = torch.empty(case["seqs"], n_q, d, device="cuda", dtype=dt)
    weights = s["w"].clone() if case["weights"] else None
    full = s["cache_grid"].full
    for i, (ids, table, there) in enumerate(s["groups"]):
        n, nb = table.shape
        k, v = [_held(*(x[table.view(-1)] for x in s["cache"][c]), full[table.view(-1)]).view(n, nb * BLOCK, h, d) for c in range(2)]
        q = s["q"][ids].float().view(n * h, n_q // h, d)
        sc = torch.bmm(q, k.permute(0, 2, 3, 1).reshape(n * h, d, nb * BLOCK)) / math.sqrt(d)
        sc = sc.view(n, n_q, nb * BLOCK).masked_fill_(~there.view(n, 1, -1), float("-inf"))
        p, l = _softmax_parts(sc)
        o = torch.bmm(p.view(n * h, n_q // h, -1), v.permute(0, 2, 1, 3).reshape(n * h, nb * BLOCK, d))
        out[ids] = (o.view(n, n_q, d) / l).to(dt)
        if case["weights"]:
            w = (p / l).view(n, h, n_q // h, -1).sum(2)                        # [sequence, head, token]
            weights[s["w_at"][i]] += w.permute(1, 0, 2)[:, there]
    return (out, weights) if case["weights"] else out


def _plain_evict(case, s):
    h, d, dt = case["n_kv"], case["d"], DTYPES[case["dtype"]]
    keep, recent, layers = case["keep"], case["recent"], case["layers"]
    at = wat = 0
    out, wout = [], []
    for n in s["new"]:
        units = 2 * layers * h
        x = s["staging"][at:at + units * n * d].view(layers, 2, h, n, d)
        w = s["weights"][wat:wat + layers * h * n].view(layers, h, n)
        at += x.numel()
        wat += w.numel()
        nb, shut = (n + BLOCK - 1) // BLOCK, n // BLOCK * BLOCK
        b = torch.nn.functional.pad(x.float(), (0, 0, 0, nb * BLOCK - n)).view(units * nb, BLOCK, 1, d)
        q, a = _quantise(b)
        if n <= keep:
            vals = (q * (a / 127.0)).view(layers, 2, h, nb * BLOCK, d)[:, :, :, :n]
            out.append(torch.cat([vals[:, :, :, :shut], x[:, :, :, shut:].float()], dim=3).to(dt).reshape(-1))
            wout.append(w.reshape(-1))
            continue
        # in units of 1 / 127: exact in 32 bits for 16-bit inputs
        vals = (q * a).view(layers, 2, h, nb * BLOCK, d)[:, :, :, :n]
        vals = torch.cat([vals[:, :, :, :shut], x[:, :, :, shut:].float() * 127.0], dim=3)
        best = torch.sort(w[:, :, :n - recent], dim=-1, descending=True, stable=True)[1][:, :, :keep - recent].sort(dim=-1)[0]
        ids = torch.cat([best, torch.arange(n - recent, n, device="cuda").expand(layers, h, recent)], dim=-1)
        kept = torch.gather(vals, 3, ids.view(layers, 1, h, keep, 1).expand(layers, 2, h, keep, d))
        nb, shut = (keep + BLOCK - 1) // BLOCK, keep // BLOCK * BLOCK
        b = torch.nn.functional.pad(kept, (0, 0, 0, nb * BLOCK - keep)).view(units * nb, BLOCK, 1, d)
        q, a = _quantise(b)
        blocks = (q * (a / 127.0 / 127.0)).view(layers, 2, h, nb * BLOCK, d)
        out.append(torch.cat([blocks[:, :, :, :shut], kept[:, :, :, shut:] / 127.0], dim=3).to(dt).reshape(-1))
        wout.append(torch.gather(w, 2, ids).reshape(-1))
    return torch.cat(out), torch.cat(wout)


# ------------------------------------------------------------------------------------------- the framework's operators
def _prepare_own(case, x):
    import paper_2503_06433_amd as ss
    new, old, h, d = x["new"], x["old"], case["n_kv"], case["d"]
    codes = {"f32": ss.SS_F32, "bf16": ss.SS_BF16, "f16": ss.SS_F16}
    lens = [n + o for n, o in zip(new, old)]
    pages = sum((n + BLOCK - 1) // BLOCK for n in lens)
    model = ss.ModelCfg(case["n_q"] * d, case["n_q"], h, d, 64, case["layers"], 0, 1e-5, 10000.0, codes[case["dtype"]], BLOCK)
    ctx = ss.Context(model, ss.RuntimeCfg(pages, 0, 0, 0, max(lens)))
    desc = ss.ShardDesc(ss.SS_PP, 1, 0, 0, case["layers"])
    ctx.kv8_enable(desc, max_seqs=case["seqs"], weights=case["weights"] or case["op"] == "evict")
    s = {"ctx": ctx, "desc": desc, "ids": list(range(case["seqs"])), "new": new, "old": old, "lens": lens}
    dt, es = DTYPES[case["dtype"]], case["layers"] * 2 * h * d
    if case["op"] == "evict":
        s["staging"] = _staging(new, x["k"], x["v"])
        t, parts = 0, []
        for n in new:
            parts.append(x["w"][:, :, t:t + n].reshape(-1))
            t += n
        s["weights"] = torch.cat(parts)
        kept = [min(n, case["keep"]) for n in new]
        s["out"] = torch.empty(es * sum(kept), device="cuda", dtype=dt)
        s["w_out"] = torch.empty(case["layers"] * h * sum(kept), device="cuda")
        s["keep"] = [case["keep"]] * case["seqs"]
        return s
    have = [i for i in s["ids"] if old[i]]
    if have:
        ctx.kv_import_dev(desc, have, [old[i] for i in have], _staging([old[i] for i in have], [x["k_old"]], [x["v_old"]]),
                          torch.cuda.current_stream().cuda_stream)
    for name in ("q", "k", "v", "w"):
        if name in x:
            s[name] = x[name]
    if case["op"] != "write":
        s["attn"] = torch.empty_like(x["q"])
    if case["op"] != "decode":
        s["out"] = torch.empty(es * sum(lens), device="cuda", dtype=dt)
    if case["weights"]:
        s["w_out"] = torch.empty_like(x["w"])
    torch.cuda.synchronize()
    return s


def _run_own(s):
    import paper_2503_06433_amd as ss
    case, ctx, desc, ids = s["case"], s["ctx"], s["desc"], s["ids"]
    st = torch.cuda.current_stream().cuda_stream
    if case["op"] == "decode":
        if not case["weights"]:
            ctx.kv8_attn_decode(desc, 0, ids, [o - 1 for o in s["old"]], s["q"], None, None, s["attn"], st)
            return s["attn"]
        ctx.kv8_weights(desc, ss.SS_IN, ids, s["w"], st)
        ctx.kv8_attn_decode(desc, 0, ids, [o - 1 for o in s["old"]], s["q"], None, None, s["attn"], st)
        ctx.kv8_weights(desc, ss.SS_OUT, ids, s["w_out"], st)
        return s["attn"], s["w_out"]
    if case["op"] == "evict":
        ctx.kv_import_dev(desc, ids, s["new"], s["staging"], st)
        ctx.kv8_weights(desc, ss.SS_IN, ids, s["weights"], st)
        ctx.kv8_evict(desc, ids, s["keep"], case["recent"], st)
        ctx.kv_export_dev(desc, ids, s["out"], st)
        ctx.kv8_weights(desc, ss.SS_OUT, ids, s["w_out"], st)
        ctx.kv_free(desc, ids)
        return s["out"], s["w_out"]
    if case["op"] == "write":
        ctx.kv8_write(desc, 0, ids, s["new"], s["old"], s["k"], s["v"], st)
        ctx.kv_export_dev(desc, ids, s["out"], st)
        return s["out"]
    ctx.kv8_attn_prefill(desc, 0, ids, s["new"], s["old"], s["q"], s["k"], s["v"], s["attn"], st)
    ctx.kv_export_dev(desc, ids, s["out"], st)
    return s["attn"], s["out"]


# ------------------------------------------------------------------------------------------------------------- calls
def prepare(case, seed):
    x = _inputs(case, seed)
    s = _prepare_own(case, x) if own else _prepare_plain(case, x)
    s["case"] = case
    return s


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["op"] == "write":
        return _plain_export(case, s, *_plain_write(case, s))
    return {"prefill": _plain_prefill, "decode": _plain_decode, "evict": _plain_evict}[case["op"]](case, s)


# ------------------------------------------------------------------------------------------------ from the definition
def exact(case, seed):
    """The same in 64 bits, sequence by sequence and block by block."""
    x = _inputs(case, seed)
    new, old, h, d, n_q = x["new"], x["old"], case["n_kv"], case["d"], case["n_q"]
    per = n_q // h

    def units(t):
        """Tokens [n, heads, d] from position 0 on -> 127 times what the cache holds of them: whole numbers times the block's
        largest magnitude, exact in 64 bits, so that a number on half a step is seen to be there when it is rounded again."""
        t = t.double()
        shut = t.shape[0] // 16 * 16
        b = t[:shut].reshape(-1, 16, t.shape[1], d)
        top = b.abs().max(dim=3)[0].max(dim=1)[0][:, None, :, None]
        # rounded to the nearest, halves to even, as torch.round does
        whole = torch.round(torch.where(top == 0, torch.zeros_like(b), b * 127 / top))
        return torch.cat([(whole * top).reshape(shut, t.shape[1], d), t[shut:] * 127])

    def blocks(t):
        return units(t) / 127

    def cached(sq, o0, n0):
        ks, vs = [], []
        for lst, name in ((ks, "k"), (vs, "v")):
            lst.append(x[name + "_old"][o0:o0 + old[sq]])
            if case["op"] != "decode":
                lst.append(x[name][n0:n0 + new[sq]])
        return blocks(torch.cat(ks)), blocks(torch.cat(vs))

    out, attn, wts = [], [], []
    o0 = n0 = w0 = 0
    for sq in range(case["seqs"]):
        if case["op"] == "evict":
            n, keep, recent = new[sq], case["keep"], case["recent"]
            wk = []
            for layer in range(case["layers"]):
                w = x["w"][layer, :, n0:n0 + n]
                pos = torch.arange(n, device="cuda").expand(h, n)
                if n > keep:
                    old_w = w[:, :n - recent]
                    rank = torch.argsort(-old_w.double(), dim=1, stable=True)[:, :keep - recent]
                    mark = torch.zeros(h, n, dtype=torch.bool, device="cuda")
                    mark.scatter_(1, rank, True)
                    mark[:, n - recent:] = True
                    pos = torch.nonzero(mark)[:, 1].view(h, keep)
                for name in ("k", "v"):
                    held = units(x[name][layer][n0:n0 + n])
                    if n > keep:
                        held = units(torch.stack([held[pos[g], g] for g in range(h)], dim=1)) / 127
                    held = held / 127
                    out.append(held.permute(1, 0, 2).reshape(-1))
                wk.append(torch.stack([w[g, pos[g]] for g in range(h)]).double().reshape(-1))
            wts += wk
            n0 += n
            continue
        k, v = cached(sq, o0, n0)
        ln = k.shape[0]
        if case["op"] != "decode":
            out += [k.permute(1, 0, 2).reshape(-1), v.permute(1, 0, 2).reshape(-1)]
        if case["op"] in ("decode", "prefill"):
            if case["op"] == "decode":
                q, first = x["q"][sq:sq + 1].double(), ln - 1
            else:
                q, first = x["q"][n0:n0 + new[sq]].double(), old[sq]
            n = q.shape[0]
            o = torch.empty(n, n_q, d, device="cuda", dtype=torch.float64)
            wsum = torch.zeros(h, ln, device="cuda", dtype=torch.float64)
            hidden = torch.ones(n, ln, dtype=torch.bool, device="cuda").triu(first + 1)
            for g in range(h):
                for a in range(g * per, (g + 1) * per):
                    z = q[:, a] @ k[:, g].t().contiguous() * d ** -0.5
                    z[hidden] = -math.inf
                    z = torch.exp(z - z.max(dim=1, keepdim=True)[0])
                    z /= z.sum(dim=1, keepdim=True)
                    o[:, a] = z @ v[:, g].contiguous()
                    if case["weights"]:
                        wsum[g] += z[0]
            attn.append(o)
            if case["weights"]:
                wts.append(x["w"][w0:w0 + h * ln].double() + wsum.reshape(-1))
                w0 += h * ln
        o0 += old[sq]
        n0 += new[sq]
    if case["op"] == "evict":
        return torch.cat(out), torch.cat(wts)
    if case["op"] == "write":
        return torch.cat(out)
    if case["op"] == "prefill":
        return torch.cat(attn), torch.cat(out)
    return (torch.cat(attn), torch.cat(wts)) if case["weights"] else torch.cat(attn)
