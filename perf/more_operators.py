"""Operators around drafted trees and cache eviction, in plain torch and through the library.

A case is one call on the tensors of one decoder layer:

* "tree"    attention of the tokens of a drafted tree over the paged INT2 cache and their own paths (int2kv_tree_attention):
            whole trees, or (`grown` tokens already there) their next level;
* "weights" attention weight that every cached token receives, added to a running sum (int2kv_token_weights): one token a
            sequence, the last tokens of a prompt, whole prompts;
* "select"  the tokens that stay: the first, the last and those of the largest weights (int2kv_select_tokens);
* "move"    the kept tokens' rows and weights into other blocks (int2kv_move_tokens).

Caches hold group-quantized N(0, 1) rows (centered keys and values in their rotated bases), written here in the documented
record layout. Lengths and the trees' levels are a property of the case; everything else is drawn from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128         # head dimension
PAGE = 16       # tokens of a cache block
SCALE = 1.0 / math.sqrt(D)
RECORD = {32: 1536, 128: 1152}
DECAY = 0.9375  # of the running sums of weights
TREE_MOST = 256
BASE = {
    "tree": dict(batch=1, n=1, grown=0, width=4, absent=0, ctx_lo=0, ctx_hi=0, q_heads=32, kv_heads=8, group=32, fused=False),
    "weights": dict(batch=1, n_lo=1, n_hi=1, ctx_lo=1, ctx_hi=1, q_heads=32, kv_heads=8, group=32, first=False),
    "select": dict(batch=1, ctx_lo=1, ctx_hi=1, kv_heads=8, budget=1, sink=0, recent=0),
    "move": dict(batch=1, ctx_lo=1, ctx_hi=1, kv_heads=8, group=32, budget=1, weights=True),
}


def _case(name, kind, **kw):
    return {"name": name, "kind": kind, **BASE[kind], **kw} if name else {"kind": kind, **BASE[kind], **kw}


def listed():
    return [
        # a single user's chat: a small tree of drafted tokens scored by the target model
        _case("tree-b1-1k", "tree", n=21, width=4, ctx_lo=1011, ctx_hi=1011),
        # a ragged serving batch, trees of one shape whose last places are empty, five query heads per KV head
        _case("tree-b24-ragged", "tree", batch=24, n=32, width=6, absent=5, ctx_lo=512, ctx_hi=16384, q_heads=40),
        # the next level of growing trees of the draft model, its rows where the layer's projection left them
        _case("tree-level-b8", "tree", batch=8, n=8, grown=41, width=8, ctx_lo=300, ctx_hi=9000, group=128, fused=True),
        # large trees on long contexts
        _case("tree-b4-200", "tree", batch=4, n=200, width=14, ctx_lo=20011, ctx_hi=32768),
        # a decode step of a single user's chat: latency
        _case("weights-b1-1k", "weights", ctx_lo=1011, ctx_hi=1011),
        # a decode step of the ragged serving batch
        _case("weights-b64-ragged", "weights", batch=64, ctx_lo=512, ctx_hi=32768, q_heads=40),
        # the last tokens of long prompts vote on the rest of them, from no sum yet
        _case("weights-last64-of-16k", "weights", batch=2, n_lo=64, n_hi=64, ctx_lo=15001, ctx_hi=16384, group=128, first=True),
        # whole prompts of odd lengths; the largest
        _case("weights-prompt-4x4k", "weights", batch=4, n_lo=3001, n_hi=4096, ctx_lo=0, ctx_hi=0),
        # a chat that outgrew its budget
        _case("select-b1-2k", "select", ctx_lo=2531, ctx_hi=2531, budget=2048, sink=4, recent=256),
        # a serving batch cut to an eighth of its longest contexts
        _case("select-b64-ragged", "select", batch=64, ctx_lo=512, ctx_hi=32768, budget=4096, sink=64, recent=256),
        # the same chat's rows
        _case("move-b1-2k", "move", ctx_lo=2531, ctx_hi=2531, budget=2048),
        # the batch's rows
        _case("move-b64-ragged", "move", batch=64, ctx_lo=512, ctx_hi=32768, budget=4096),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "weights", "weights", "select", "move"])
    group = rng.choice([32, 128])
    q_heads, kv_heads = rng.choice([(32, 8), (40, 8), (32, 4), (16, 8), (4, 1)])
    batch = _log_int(rng, 1, 64)
    if kind == "tree":
        n = _log_int(rng, 1, min(TREE_MOST, 1024 // batch))
        ctx_hi = max(16, min(_log_int(rng, 16, max(16, 262144 // batch)), 32768, 600_000_000 // (batch * n * q_heads)))
        grown = rng.randrange(0, TREE_MOST - n + 1) if rng.random() < 0.4 else 0
        return _case("", kind, batch=batch, n=n, grown=min(grown, 4 * n), width=rng.randint(1, 16),
                     absent=rng.randrange(0, n) // 3 if rng.random() < 0.3 else 0,
                     ctx_lo=int(ctx_hi * rng.choice([1.0, 0.5, 0.0])), ctx_hi=ctx_hi, q_heads=q_heads, kv_heads=kv_heads,
                     group=group, fused=rng.random() < 0.4)
    if kind == "weights":
        n = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, 4096 // batch))
        ctx_hi = max(16, min(_log_int(rng, 16, max(16, 524288 // batch)), 32768, 400_000_000 // (batch * n * q_heads)))
        return _case("", kind, batch=batch, n_lo=max(1, int(n * rng.choice([1.0, 0.3]))), n_hi=n,
                     ctx_lo=int(ctx_hi * rng.choice([1.0, 0.5, 0.0])), ctx_hi=ctx_hi, q_heads=q_heads, kv_heads=kv_heads,
                     group=group, first=rng.random() < 0.3)
    ctx_hi = _log_int(rng, 64, min(32768, 1048576 // batch))
    budget = _log_int(rng, 16, ctx_hi)
    lo = max(1, int(ctx_hi * rng.choice([1.0, 0.5, 0.1])))
    if kind == "select":
        sink = rng.randint(0, budget // 4)
        return _case("", kind, batch=batch, ctx_lo=lo, ctx_hi=ctx_hi, kv_heads=kv_heads, budget=budget, sink=sink,
                     recent=rng.randint(0, budget - sink))
    return _case("", kind, batch=batch, ctx_lo=lo, ctx_hi=ctx_hi, kv_heads=kv_heads, group=group, budget=budget,
                 weights=rng.random() < 0.6)


# ---------------------------------------------------------------------------------------------
# Inputs

def _lens(case):
    """(new tokens, cached tokens) of each sequence: a property of the case, the same for every seed. Where the cache holds
    the new tokens too ("weights"), its lengths count them."""
    kind = case["kind"]
    lo, hi = (case["n_lo"], case["n_hi"]) if kind == "weights" else (case.get("n", 0),) * 2
    r = random.Random("%d %d %d" % (case["batch"], hi, case["ctx_hi"]))
    n = [r.randint(lo, hi) for _ in range(case["batch"])]
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["batch"])]
    if kind == "weights":
        ctx = [c if m == 1 and c else c + m for m, c in zip(n, ctx)]
    return n, ctx


def _gen(seed, salt):
    return torch.Generator("cuda").manual_seed(int(seed) * 64 + salt)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _rotations(seed, heads):
    """Haar-random orthogonal matrices, fp32 [heads, 128, 128]: QR of a Gaussian with the signs of diag(R) folded in."""
    g = torch.Generator().manual_seed(int(seed))
    q, r = torch.linalg.qr(torch.randn((heads, D, D), generator=g, dtype=torch.float64))
    return (q * torch.sign(torch.diagonal(r, dim1=1, dim2=2))[:, None, :]).float().contiguous().cuda()


def _offsets(seed, heads):
    """Constant key offsets: three channels per KV head at 10 to 30 (what key centering removes)."""
    r = random.Random(int(seed))
    off = torch.zeros((heads, D))
    for h in range(heads):
        for c in r.sample(range(D), 3):
            off[h, c] = r.uniform(10.0, 30.0)
    return off.cuda()


def _records(rows_k, rows_v, group):
    """Packed records uint8 [n, H, bytes] of n blocks of 16 rows: fp32 [n, H, 16, 128]."""
    n, H = rows_k.shape[:2]

    def parts(x):
        g = x.reshape(n, H, PAGE, D // group, group)
        mn, mx = g.amin(-1), g.amax(-1)
        s, z = ((mx - mn) / 3.0).half(), mn.half()
        codes = torch.clamp(torch.round((g - z.float()[..., None]) / s.float()[..., None]), 0, 3).to(torch.int32)
        c = codes.reshape(n, H, PAGE, 8, 16)
        half = (c << (2 * torch.arange(8, device=x.device, dtype=torch.int32))[:, None]).sum(-2).to(torch.int16)
        return half, s, z

    flat = lambda t: t.contiguous().view(torch.uint8).reshape(n, H, -1)  # noqa: E731
    kh, ks, kz = parts(rows_k)
    vh, vs, vz = parts(rows_v)
    return torch.cat([flat(kh), flat(vh.transpose(2, 3)), flat(torch.stack([ks, kz], -1)), flat(vs.transpose(2, 3)),
                      flat(vz.transpose(2, 3))], dim=-1)


def _random_pool(seed, blocks, heads, group, empty=0):
    """`blocks` blocks of drawn rows, and `empty` zero ones behind them."""
    pool = torch.empty((blocks + empty, heads, RECORD[group]), dtype=torch.uint8, device="cuda")
    pool[blocks:].zero_()
    g, step = _gen(seed, 1), max(1, 16384 // heads)
    for i in range(0, blocks, step):
        n = min(step, blocks - i)
        pool[i:i + n] = _records(_randn(g, n, heads, PAGE, D), _randn(g, n, heads, PAGE, D), group)
    return pool


def _table(lens, seed, base=0):
    """Block table int32 [B, pages of the longest] over permuted blocks base .., and how many there are."""
    pages = [-(-c // PAGE) for c in lens]
    blocks = max(1, sum(pages))
    phys = base + torch.randperm(blocks, generator=torch.Generator().manual_seed(int(seed))).to(torch.int32)
    table, at = torch.zeros((len(lens), max(1, max(pages))), dtype=torch.int32), 0
    for b, m in enumerate(pages):
        table[b, :m] = phys[at:at + m]
        at += m
    return table.cuda(), blocks


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _prepare_tree(case, seed):
    n, ctx = _lens(case)
    B, H, Hq, T, width = case["batch"], case["kv_heads"], case["q_heads"], case["grown"] + case["n"], case["width"]
    g, r, off, total = _gen(seed, 2), random.Random(int(seed)), _offsets(seed, H), sum(n)
    table, blocks = _table(ctx, seed)
    # levels of `width` tokens, each with a parent in the level before; the last places of a tree may be empty
    parents = [(t // width - 1) * width + r.randrange(width) if t >= width else -1 for _ in range(B) for t in range(T)]
    for b in range(B):
        for t in range(T - case["absent"], T):
            parents[b * T + t] = -2
    k = (_randn(g, B * T, H, D) + off).to(torch.bfloat16)
    v = _randn(g, B * T, H, D).to(torch.bfloat16)
    if case["fused"]:  # where the layer's projection left them, beside its queries
        qkv = torch.zeros((B * T, Hq + 2 * H, D), dtype=torch.bfloat16, device="cuda")
        qkv[:, Hq:Hq + H], qkv[:, Hq + H:] = k, v
        k, v = qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    return dict(q=(2.0 * _randn(g, total, Hq, D)).to(torch.bfloat16), parents=_i32(parents), k=k, v=v, mu=off, table=table,
                starts=_i32([sum(n[:b]) for b in range(B + 1)]), trees=_i32([b * T for b in range(B + 1)]), lens=_i32(ctx),
                max_ctx=max(ctx), pool=_random_pool(seed, blocks, H, case["group"]), R_k=_rotations(2 * seed + 1, H),
                R_v=_rotations(2 * seed + 2, H), out=torch.zeros((total, Hq, D), dtype=torch.bfloat16, device="cuda"))


def _drawn_weights(g, B, H, L):
    """Running sums as decoding leaves them: a few tokens hold most of the weight, equal values occur."""
    return torch.exp(2.0 * _randn(g, B, H, L) - 4.0).to(torch.bfloat16).float()


def _prepare_weights(case, seed):
    n, ctx = _lens(case)
    B, H, Hq = case["batch"], case["kv_heads"], case["q_heads"]
    g, total = _gen(seed, 3), sum(n)
    table, blocks = _table(ctx, seed)
    w = None if case["first"] else _drawn_weights(g, B, H, max(ctx))
    return dict(q=(2.0 * _randn(g, total, Hq, D)).to(torch.bfloat16), starts=_i32([sum(n[:b]) for b in range(B + 1)]), table=table,
                lens=_i32(ctx), n=n, ctx=ctx, max_q=max(n), max_ctx=max(ctx), pool=_random_pool(seed, blocks, H, case["group"]),
                R_k=_rotations(2 * seed + 1, H), w=w, w_out=torch.zeros((B, H, max(ctx)), dtype=torch.float32, device="cuda"))


def _prepare_select(case, seed):
    _, ctx = _lens(case)
    B, H, keep = case["batch"], case["kv_heads"], case["budget"]
    return dict(w=_drawn_weights(_gen(seed, 4), B, H, max(ctx)), lens=_i32(ctx), max_ctx=max(ctx),
                kept=torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda"),
                kept_lens=torch.zeros(B, dtype=torch.int32, device="cuda"))


def _prepare_move(case, seed):
    _, ctx = _lens(case)
    B, H, keep = case["batch"], case["kv_heads"], case["budget"]
    g, lens = _gen(seed, 5), [min(c, keep) for c in ctx]
    table, blocks = _table(ctx, seed)
    out_table, out_blocks = _table(lens, seed + 1, blocks)
    kept = torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda")
    for b, (c, m) in enumerate(zip(ctx, lens)):  # any m of the c tokens, in order
        kept[b, :, :m] = torch.rand((H, c), generator=g, device="cuda").argsort(1)[:, :m].sort(1)[0].to(torch.int32)
    w = _drawn_weights(g, B, H, max(ctx)) if case["weights"] else None
    return dict(pool=_random_pool(seed, blocks, H, case["group"], out_blocks), table=table, out_table=out_table, blocks=blocks,
                kept=kept, kept_lens=_i32(lens), max_kept=max(lens), w=w,
                w_out=torch.zeros((B, H, keep), dtype=torch.float32, device="cuda") if case["weights"] else None)


def prepare(case, seed):
    s = {"tree": _prepare_tree, "weights": _prepare_weights, "select": _prepare_select, "move": _prepare_move}[case["kind"]](case, seed)
    return {**s, "case": case}


# ---------------------------------------------------------------------------------------------
# The plain forms

def _unpack(rec, group, values=True):
    """Dequantized rows [..., 16, 128] (keys, values) of packed records [..., bytes]."""
    ng, lead = D // group, rec.shape[:-1]
    shift = 2 * torch.arange(8, device=rec.device, dtype=torch.int16)

    def rows(half, s, z):  # half [..., 16, 16]: channel 16 p + m of a token at bits 2 p of its half m
        codes = ((half[..., None, :] >> shift[:, None]) & 3).reshape(*lead, PAGE, ng, group)
        return (codes.float() * s.float()[..., None] + z.float()[..., None]).reshape(*lead, PAGE, D)

    kh = rec[..., :512].contiguous().view(torch.int16).reshape(*lead, PAGE, 16)
    km = rec[..., 1024:1024 + 64 * ng].contiguous().view(torch.float16).reshape(*lead, PAGE, ng, 2)
    k = rows(kh, km[..., 0], km[..., 1])
    if not values:
        return k, None
    vh = rec[..., 512:1024].contiguous().view(torch.int16).reshape(*lead, 16, PAGE).transpose(-1, -2)
    vm = rec[..., 1024 + 64 * ng:].contiguous().view(torch.float16).reshape(*lead, 2, ng, PAGE).transpose(-1, -2)
    return k, rows(vh, vm[..., 0, :, :], vm[..., 1, :, :])


def _paths(parents, B, T):
    """[B, T, T]: whether token t lies on the path of token i (row), itself included; absent tokens have no path."""
    at = parents.reshape(B, T).long()
    step = ((at[..., None] == torch.arange(T, device="cuda")) | torch.eye(T, dtype=torch.bool, device="cuda")).float()
    for _ in range(max(1, (T - 1).bit_length())):
        step = (torch.matmul(step, step) > 0).float()
    return (step > 0) & (at >= -1)[..., None]


def _plain_tree(s):
    """All sequences at once, padded to the longest: rows are (new token, query head of the KV head's group)."""
    case = s["case"]
    B, H, G, n = case["batch"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["n"]
    T = case["grown"] + n
    q = s["q"].float().reshape(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    L = s["table"].shape[1] * PAGE
    k, v = _unpack(s["pool"][s["table"].long()], case["group"])                    # [B, pages, H, 16, 128]
    live = torch.arange(L, device="cuda") < s["lens"][:, None]
    k, v = (torch.where(live[:, None, :, None], x.transpose(1, 2).reshape(B, H, L, D), 0.0) for x in (k, v))
    kn = s["k"].float().reshape(B, T, H, D).transpose(1, 2) - s["mu"][:, None]
    vn = s["v"].float().reshape(B, T, H, D).transpose(1, 2).contiguous()
    a = torch.cat([torch.matmul(torch.matmul(q, s["R_k"]), k.transpose(-1, -2).contiguous()),
                   torch.matmul(q, kn.transpose(-1, -2).contiguous())], -1)
    path = _paths(s["parents"], B, T)[:, case["grown"]:]                             # [B, n, T]
    seen = torch.cat([live[:, None] & path.any(-1, keepdim=True), path], -1).repeat_interleave(G, 1)[:, None]
    a = torch.where(seen, a * SCALE, -math.inf)
    p = torch.exp(a - a.amax(-1, keepdim=True).clamp(min=-1e30))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.matmul(torch.matmul(p[..., :L], v), s["R_v"].transpose(-1, -2).contiguous()) + torch.matmul(p[..., L:], vn)
    return {"out": o.reshape(B, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(B * n, H * G, D).to(torch.bfloat16)}


def _plain_weights(s):
    """A sequence after the other, 512 new tokens at a time."""
    case = s["case"]
    H, G, out, at = case["kv_heads"], case["q_heads"] // case["kv_heads"], s["w_out"], 0
    for b, (n, c) in enumerate(zip(s["n"], s["ctx"])):
        rec = s["pool"][s["table"][b, :-(-c // PAGE)].long()]
        k = _unpack(rec, case["group"], False)[0].transpose(0, 1).reshape(H, -1, D)[:, :c].transpose(1, 2).contiguous()
        t = torch.arange(c, device="cuda")
        got = torch.zeros((H, c), device="cuda") if s["w"] is None else DECAY * s["w"][b, :, :c]
        for i0 in range(0, n, 512):
            m = min(512, n - i0)
            q = s["q"][at + i0:at + i0 + m].float().reshape(m, H, G, D).transpose(0, 1).reshape(H, m * G, D)
            a = torch.matmul(torch.matmul(q, s["R_k"]), k) * SCALE
            limit = (c - n + i0 + torch.arange(m, device="cuda") + 1).repeat_interleave(G)
            a = torch.where(t < limit[:, None], a, -math.inf)
            p = torch.exp(a - a.amax(-1, keepdim=True))
            got = got + (p / p.sum(-1, keepdim=True)).sum(1)
        out[b, :, :c] = got
        at += n
    return {"weights": out}


def _plain_select(s):
    case = s["case"]
    B, H, L = s["w"].shape
    t, lens, keep = torch.arange(L, device="cuda"), s["lens"][:, None].long(), case["budget"]
    forced = (t < case["sink"]) | (t >= lens - case["recent"])
    w = torch.where(forced[:, None], math.inf, s["w"])
    w = torch.where((t < lens)[:, None], w, -math.inf)
    first = torch.sort(w, dim=-1, descending=True, stable=True)[1][..., :keep]       # ties: the lower index
    count = lens.clamp(max=keep)
    j = torch.arange(first.shape[-1], device="cuda")
    ordered = torch.sort(torch.where(j < count[:, None], first, L), dim=-1)[0].to(torch.int32)
    s["kept"][..., :first.shape[-1]] = torch.where(j < count[:, None], ordered, s["kept"][..., :first.shape[-1]])
    s["kept_lens"].copy_(count[:, 0])
    return {"kept": s["kept"], "kept_lens": s["kept_lens"]}


def _plain_move(s):
    """Rows taken apart by fields, gathered and put together again; rows behind the last kept one stay."""
    case = s["case"]
    ng, H, pool = D // case["group"], case["kv_heads"], s["pool"]
    for b in range(case["batch"]):
        m = int(min(s["max_kept"], case["budget"], s["kept"].shape[-1]))
        pages = s["out_table"].shape[1]
        kept = torch.zeros((H, pages * PAGE), dtype=torch.long, device="cuda")
        kept[:, :m] = s["kept"][b, :, :m]
        real = torch.arange(pages * PAGE, device="cuda") < s["kept_lens"][b]
        kept = torch.where(real, kept, 0)
        block, tok, head = s["table"][b].long()[kept // PAGE], kept % PAGE, torch.arange(H, device="cuda")[:, None]
        k = pool[..., :512].unflatten(-1, (PAGE, 32))[block, head, tok]                                    # [H, tokens, 32]
        v = pool[..., 512:1024].unflatten(-1, (16, PAGE, 2))[block, head, :, tok]                          # [H, tokens, 16, 2]
        km = pool[..., 1024:1024 + 64 * ng].unflatten(-1, (PAGE, 4 * ng))[block, head, tok]
        vm = pool[..., 1024 + 64 * ng:].unflatten(-1, (2 * ng, PAGE, 2))[block, head, :, tok]
        paged = lambda x: x.reshape(H, pages, PAGE, *x.shape[2:])  # noqa: E731
        rec = torch.cat([paged(k).flatten(2), paged(v).transpose(2, 3).flatten(2), paged(km).flatten(2), paged(vm).transpose(2, 3).flatten(2)],
                        -1).transpose(0, 1)                                                                # [pages, H, bytes]
        at = s["out_table"][b].long()
        keep = _byte_tokens(case["group"]) < (s["kept_lens"][b] - PAGE * torch.arange(pages, device="cuda"))[:, None]
        pool[at] = torch.where(keep[:, None], rec, pool[at])
        if s["w"] is not None:
            n = s["w_out"].shape[-1]
            got = torch.gather(s["w"][b], 1, kept[:, :n].clamp(max=s["w"].shape[-1] - 1))
            s["w_out"][b, :, :got.shape[1]] = torch.where(real[:n], got, s["w_out"][b, :, :got.shape[1]])
    return {"records": pool[s["blocks"]:], **({} if s["w"] is None else {"weights": s["w_out"]})}


def _byte_tokens(group):
    """The token (of its block) that each byte of a record belongs to."""
    ng = D // group
    o = torch.arange(RECORD[group], device="cuda")
    return torch.where(o < 512, o // 32, torch.where(o < 1024, o % 32 // 2, torch.where(o < 1024 + 64 * ng, (o - 1024) // (4 * ng),
                                                                                     o % 32 // 2)))


# ---------------------------------------------------------------------------------------------
# The library's calls

def _cache(K, s):
    """The cache's handle, which a program makes once beside its pool."""
    if "cache" not in s:
        pool = s["pool"]
        s["cache"] = K.Int2KVCache(pool.shape[0], pool.shape[1], pool=pool, group_size=s["case"]["group"])
    return s["cache"]


def _workspace(s, need):
    if "ws" not in s:
        s["ws"] = torch.empty(max(256, need()), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _own_tree(K, s):
    case = s["case"]
    T, n = case["grown"] + case["n"], case["n"]
    ws = _workspace(s, lambda: K.int2kv_tree_attention_workspace_bytes(case["batch"], case["q_heads"], case["kv_heads"],
                                                                       s["q"].shape[0], n, T, s["max_ctx"]))
    return {"out": K.int2kv_tree_attention(_cache(K, s), s["q"], s["starts"], n, s["parents"], s["k"], s["v"], s["mu"], s["table"],
                                           s["lens"], s["max_ctx"], s["R_k"], s["R_v"], tree_starts=s["trees"], max_tree=T,
                                           out=s["out"], workspace=ws)}


def _own_weights(K, s):
    case = s["case"]
    ws = _workspace(s, lambda: K.int2kv_token_weights_workspace_bytes(case["batch"], case["q_heads"], case["kv_heads"],
                                                                      s["q"].shape[0], s["max_q"], s["max_ctx"]))
    return {"weights": K.int2kv_token_weights(_cache(K, s), s["q"], s["starts"], s["max_q"], s["table"], s["lens"], s["max_ctx"],
                                              s["R_k"], weights=s["w"], decay=DECAY, out=s["w_out"], workspace=ws)}


def _own_select(K, s):
    case = s["case"]
    K.int2kv_select_tokens(s["w"], s["lens"], s["max_ctx"], case["budget"], sink=case["sink"], recent=case["recent"],
                           kept=s["kept"], kept_lens=s["kept_lens"])
    return {"kept": s["kept"], "kept_lens": s["kept_lens"]}


def _own_move(K, s):
    K.int2kv_move_tokens(_cache(K, s), s["table"], s["kept"], s["kept_lens"], s["max_kept"], out_table=s["out_table"],
                         weights=s["w"], out_weights=s["w_out"])
    return {"records": s["pool"][s["blocks"]:], **({} if s["w"] is None else {"weights": s["w_out"]})}


def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2608_02691_amd import int2kv as K
        return {"tree": _own_tree, "weights": _own_weights, "select": _own_select, "move": _own_move}[kind](K, s)
    return {"tree": _plain_tree, "weights": _plain_weights, "select": _plain_select, "move": _plain_move}[kind](s)


# ---------------------------------------------------------------------------------------------
# What a pass cannot do without

def work(case):
    H, kind = case["kv_heads"], case["kind"]
    n, ctx = _lens(case)
    if kind == "select":
        return {"bytes": 4 * H * sum(ctx) + 4 * H * sum(min(c, case["budget"]) for c in ctx) + 8 * len(ctx), "flops": H * sum(ctx)}
    rot, token, pages = 4 * D * D, RECORD[case["group"]] // PAGE, sum(-(-c // PAGE) for c in ctx)
    if kind == "move":
        kept = sum(min(c, case["budget"]) for c in ctx)
        return {"bytes": kept * H * (2 * token + 4 + (8 if case["weights"] else 0)) + 4 * pages + 4 * (kept // PAGE), "flops": 0}
    Hq, total = case["q_heads"], sum(n)
    if kind == "weights":
        pairs = sum(m * (c - m) + m * (m + 1) // 2 for m, c in zip(n, ctx))
        return {"bytes": sum(ctx) * H * (token // 2 + (4 if case["first"] else 8)) + 4 * pages + 2 * total * Hq * D + H * rot + 8 * len(n),
                "flops": 2 * D * Hq * pairs + 2 * D * D * total * Hq}
    T, live = case["grown"] + case["n"], [t for t in range(case["grown"], case["grown"] + case["n"] - case["absent"])]
    pairs = sum(len(live) * c + sum(t // case["width"] + 1 for t in live) for c in ctx)
    return {"bytes": sum(ctx) * H * token + 4 * pages + 4 * total * Hq * D + len(n) * T * (4 * H * D + 4) + 2 * H * rot + 12 * len(n),
            "flops": 4 * D * Hq * pairs + 2 * 2 * D * D * total * Hq}


# ---------------------------------------------------------------------------------------------
# The same outputs from their definitions, in 64 bits

def _stored(pool, group, block, token, h, values):
    """Row fp64 [n, 128] (keys or values) of head h of the cache's tokens, from the record layout byte by byte."""
    ng = D // group
    rec = pool[block, h].to(torch.int64)                                             # [n, bytes]
    n = rec.shape[0]
    ch = torch.arange(D, device=pool.device)
    m, bits, grp = ch % 16, 2 * (ch // 16), ch // group
    tok = token[:, None]

    def u16(byte):
        byte = byte.expand(n, byte.shape[-1])
        return rec.gather(1, byte) + 256 * rec.gather(1, byte + 1)

    def f16(byte):
        return u16(byte).to(torch.int32).to(torch.int16).view(torch.float16).double()

    if values:
        vm = 1024 + 64 * ng + 32 * grp + 2 * tok
        return ((u16(512 + 32 * m + 2 * tok) >> bits) & 3) * f16(vm) + f16(vm + 32 * ng)
    km = 1024 + 4 * ng * tok + 4 * grp
    return ((u16(32 * tok + 2 * m) >> bits) & 3) * f16(km) + f16(km + 2)


def _exact_tree(case, s):
    (n, ctx), G, T = _lens(case), case["q_heads"] // case["kv_heads"], case["grown"] + case["n"]
    Rk, Rv, parents = s["R_k"].double(), s["R_v"].double(), s["parents"].tolist()
    outs, at = [], 0
    for b, (m, c) in enumerate(zip(n, ctx)):
        sees = torch.zeros((m, c + T), dtype=torch.bool)
        for i in range(m):
            t = case["grown"] + i
            if parents[b * T + t] < -1:
                continue
            sees[i, :c] = True
            while t >= 0:
                sees[i, c + t] = True
                t = parents[b * T + t]
        sees = sees.cuda().repeat_interleave(G, 0)
        t = torch.arange(c, device="cuda")
        block, tok, heads = s["table"][b].long()[t // PAGE], t % PAGE, []
        for h in range(case["kv_heads"]):
            kn = s["k"][b * T:(b + 1) * T, h].double() - s["mu"][h].double()
            keys = torch.cat([torch.matmul(_stored(s["pool"], case["group"], block, tok, h, False), Rk[h].t()), kn])
            values = torch.cat([torch.matmul(_stored(s["pool"], case["group"], block, tok, h, True), Rv[h].t()),
                                s["v"][b * T:(b + 1) * T, h].double()])
            a = torch.matmul(s["q"][at:at + m, h * G:(h + 1) * G].double().reshape(m * G, D), keys.t()) / math.sqrt(D)
            p = torch.nan_to_num(torch.softmax(a.masked_fill(~sees, -math.inf), -1))  # a row that sees nothing: zeros
            heads.append(torch.matmul(p, values).reshape(m, G, D))
        outs.append(torch.stack(heads, 1).reshape(m, -1, D))
        at += m
    return {"out": torch.cat(outs)}


def _exact_weights(case, s):
    G, at = case["q_heads"] // case["kv_heads"], 0
    out = torch.zeros(s["w_out"].shape, dtype=torch.float64, device="cuda")
    for b, (n, c) in enumerate(zip(s["n"], s["ctx"])):
        t = torch.arange(c, device="cuda")
        for h in range(case["kv_heads"]):
            keys = torch.matmul(_stored(s["pool"], case["group"], s["table"][b].long()[t // PAGE], t % PAGE, h, False),
                                s["R_k"][h].double().t())
            if s["w"] is not None:
                out[b, h, :c] = s["w"][b, h, :c].double() * DECAY
            for j in range(h * G, (h + 1) * G):
                a = torch.matmul(s["q"][at:at + n, j].double(), keys.t()) / math.sqrt(D)
                a = a.masked_fill(t > c - n + torch.arange(n, device="cuda")[:, None], -math.inf)
                out[b, h, :c] += torch.softmax(a, -1).sum(0)
        at += n
    return {"weights": out}


def _exact_select(case, s):
    w, lens = s["w"].cpu().numpy(), s["lens"].tolist()
    kept = np.full(tuple(s["kept"].shape), -1, np.int32)
    for b, c in enumerate(lens):
        m = min(c, case["budget"])
        t = np.arange(c)
        forced = (t < case["sink"]) | (t >= c - case["recent"])
        rest = t[~forced]
        for h in range(case["kv_heads"]):
            if m == c:
                kept[b, h, :m] = t
                continue
            best = rest[np.argsort(-w[b, h, rest], kind="stable")[:m - int(forced.sum())]]
            kept[b, h, :m] = np.sort(np.concatenate([t[forced], best]))
    return {"kept": torch.from_numpy(kept).cuda(), "kept_lens": _i32([min(c, case["budget"]) for c in lens])}


def _exact_move(case, s):
    """Every byte of a kept row by its place in the record."""
    pool, lens = s["pool"], s["kept_lens"].tolist()
    got = pool[s["blocks"]:].clone()
    meta, o = 512 // case["group"], torch.arange(RECORD[case["group"]], device="cuda")
    wide, keys = o < 512, (o >= 1024) & (o < 1024 + PAGE * meta)  # key codes and key parameters lie token by token
    step = torch.where(wide, 32, torch.where(keys, meta, 2))      # bytes from a token to the next
    tok = torch.where(wide, o // 32, torch.where(keys, (o - 1024) // meta, o % 32 // 2))
    base = o - step * tok
    weights = None if s["w"] is None else torch.zeros(s["w_out"].shape, dtype=torch.float64, device="cuda")
    for b, m in enumerate(lens):
        for p in range(-(-m // PAGE)):
            new = (PAGE * p + tok).clamp(max=m - 1)
            old = s["kept"][b][:, new].long()                                         # [H, bytes]
            src = pool[s["table"][b].long()[old // PAGE], torch.arange(case["kv_heads"], device="cuda")[:, None], base + step * (old % PAGE)]
            at = int(s["out_table"][b, p]) - s["blocks"]
            got[at] = torch.where(PAGE * p + tok < m, src, got[at])
        if weights is not None:
            weights[b, :, :m] = torch.gather(s["w"][b], 1, s["kept"][b, :, :m].long()).double()
    return {"records": got, **({} if weights is None else {"weights": weights})}


def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _exact_tree, "weights": _exact_weights, "select": _exact_select, "move": _exact_move}[case["kind"]](case, s)
