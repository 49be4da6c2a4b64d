"""Timed calls of the operators around the paged key/value cache, and their plain forms.

A served prompt's keys and values stay in a cache of pages.  One step of a batch of requests is: the plan of the step (block
tables, slots, positions and, for drafted trees, ancestors), per layer the norms and the rotation of queries and keys with the
cache's write, the attention of the new tokens over the cache, and after the drafted tokens' verification the move that closes
up the accepted ones behind the context.

A case is a dict with a `kind`:
  plan    sp_cache_plan    batch requests with contexts up to `ctx` that add up to `new` tokens each (ragged: as the lengths'
                           own seed gives them), as trees or not
  rope    sp_qk_norm_rope  `tokens` rows of a fused projection
  attn    sp_cache_attn    batch requests with contexts up to `ctx` and `new` drafted tokens each (1: ordinary decoding)
  accept  sp_cache_accept  `layers` layers' caches, up to `accept` of `new` drafted tokens stay
Sizes of heads are those of the configurations (synth/generator.py) and perf/cases.py.
"""
import math
import random

import torch

own = False


def _sp():
    import paper_2505_19578_amd as sp
    return sp


# ------------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a decoding step of a full server: one token for each of 256 requests
        dict(name="plan_decode_256", kind="plan", batch=256, ctx=8192, new=1, page=16, tree=False, ragged=False, lens=1),
        # a speculative step: trees of 32 drafted tokens
        dict(name="plan_tree_96x32", kind="plan", batch=96, ctx=16384, new=32, page=64, tree=True, ragged=False, lens=2),
        # prompts that arrive together, 1 to 8K tokens each
        dict(name="plan_prompts_40", kind="plan", batch=40, ctx=0, new=8192, page=64, tree=False, ragged=True, lens=3),
        # one request decodes one token: a launch is what its user waits for
        dict(name="rope_1", kind="rope", tokens=1, q_heads=32, kv_heads=8, head_dim=128, rotary=128, interleaved=False,
             norm=True, page=16, far=8192),
        # the drafted trees of 61 requests, the 70B shape without norms, far positions
        dict(name="rope_1952", kind="rope", tokens=1952, q_heads=64, kv_heads=8, head_dim=128, rotary=128, interleaved=False,
             norm=False, page=64, far=1000000),
        # a 32K prompt of the headline shape on its way into the prefill and the cache
        dict(name="rope_32k", kind="rope", tokens=32768, q_heads=32, kv_heads=8, head_dim=128, rotary=128, interleaved=False,
             norm=True, page=64, far=0),
        # ordinary decoding, one request: the reader of one short document
        dict(name="attn_1x4k", kind="attn", batch=1, ctx=4000, new=1, q_heads=32, kv_heads=8, head_dim=128, page=16,
             ragged=False, lens=4),
        # ordinary decoding of a batch of ragged lengths: every byte of the cache once
        dict(name="attn_64x16k", kind="attn", batch=64, ctx=16384, new=1, q_heads=32, kv_heads=8, head_dim=128, page=64,
             ragged=True, lens=5),
        # drafted trees over medium contexts, seven query heads to a KV head
        dict(name="attn_tree_12x6k", kind="attn", batch=12, ctx=6150, new=21, q_heads=28, kv_heads=4, head_dim=128, page=32,
             ragged=True, lens=6),
        # a large tree over one prompt of the headline length
        dict(name="attn_tree_1x128k", kind="attn", batch=1, ctx=131000, new=64, q_heads=64, kv_heads=8, head_dim=128,
             page=128, ragged=False, lens=7),
        # the end of a speculative step, one request, every layer
        dict(name="accept_1", kind="accept", batch=1, ctx=500, new=24, accept=5, layers=32, kv_heads=8, head_dim=128, page=16,
             lens=8),
        # and of a batch
        dict(name="accept_48", kind="accept", batch=48, ctx=700, new=40, accept=8, layers=16, kv_heads=8, head_dim=128,
             page=64, lens=9),
    ]


# query heads, KV heads, head_dim
_SHAPES = [(32, 8, 128), (28, 4, 128), (64, 8, 128), (4, 4, 64), (16, 16, 64), (32, 8, 64)]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    """One more case: any kind; sizes spread over their logarithm."""
    kind = rng.choice(["plan", "rope", "attn", "attn", "accept"])
    q_heads, kv_heads, head_dim = rng.choice(_SHAPES)
    page = rng.choice([16, 32, 64, 128, 256])
    c = dict(kind=kind, page=page)
    if kind == "plan":
        tree = rng.random() < 0.4
        c.update(batch=_log(rng, 1, 512), ctx=_log(rng, 1, 32768), new=_log(rng, 1, 256 if tree else 8192), tree=tree,
                 ragged=rng.random() < 0.7, lens=rng.randrange(1 << 30))
        c["batch"] = max(1, min(c["batch"], 327680 // (c["new"] * (8 if tree else 1))))
    elif kind == "rope":
        rotary = rng.choice([head_dim, head_dim, head_dim // 2, 0])
        c.update(tokens=_log(rng, 1, 32768), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, rotary=rotary,
                 interleaved=rng.random() < 0.3, norm=rng.random() < 0.6 or rotary == 0, far=rng.choice([0, 4096, 1000000]))
        c["tokens"] = max(1, min(c["tokens"], 32768 * 48 * 128 // ((q_heads + 2 * kv_heads) * head_dim)))
    elif kind == "attn":
        c.update(batch=_log(rng, 1, 128), ctx=_log(rng, 1, 131072), new=rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 2, 64)]),
                 q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, ragged=rng.random() < 0.6, lens=rng.randrange(1 << 30))
        c["batch"] = max(1, min(c["batch"], (1 << 29) // (c["ctx"] * kv_heads * head_dim)))
        c["new"] = max(1, min(c["new"], (1 << 29) // (c["batch"] * c["ctx"] * q_heads)))
    else:
        new = _log(rng, 2, 64)
        c.update(batch=_log(rng, 1, 64), ctx=_log(rng, 1, 1024), new=new, accept=rng.randint(1, min(16, new)),
                 layers=_log(rng, 1, 32), kv_heads=kv_heads, head_dim=head_dim, lens=rng.randrange(1 << 30))
        per = (c["ctx"] + new + page) * kv_heads * head_dim * c["layers"]
        c["batch"] = max(1, min(c["batch"], (1 << 29) // per))
    return c


# ---------------------------------------------------------------------------------------------------------------- lengths
def _lengths(c):
    """(contexts, numbers of new tokens) of a case's requests: its own, whatever the seed of the values."""
    r = random.Random(c["lens"])
    n, ctx, new = c["batch"], c["ctx"], c["new"]
    spread = c.get("ragged", True)
    cs = [ctx if not spread else r.randint(0, ctx) if r.random() < 0.8 else ctx for _ in range(n)]
    if c["kind"] == "plan" and not c["ragged"]:
        cs = [r.randint(0, ctx) for _ in range(n)]
        ts = [new] * n
    elif c["kind"] == "plan":
        ts = [r.randint(1, new) for _ in range(n)]
    else:
        ts = [new] * n if not spread else [max(1, new - r.randint(0, new // 2)) for _ in range(n)]
    cs[0] = ctx
    return cs, ts


def _pages(c):
    cs, ts = _lengths(c)
    return [-(-(x + y) // c["page"]) for x, y in zip(cs, ts)]


# ----------------------------------------------------------------------------------------------------------------- inputs
def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _parents(ts, seed):
    """Drafted trees: token 0 is the root, every other one hangs below one of the tokens shortly before it."""
    r, out = random.Random(seed), []
    for t in ts:
        out += [-1] + [r.randint(max(0, i - 8), i - 1) for i in range(1, t)]
    return out


def _ancestor_words(parents, ts, words):
    out, at = [], 0
    for t in ts:
        m = []
        for i in range(t):
            p = parents[at + i]
            m.append((m[p] if p >= 0 else 0) | (1 << i))
        out += m
        at += t
    rows = [[(x >> (64 * w)) & ((1 << 64) - 1) for w in range(words)] for x in out]
    return torch.tensor([[x - (1 << 64) if x >> 63 else x for x in row] for row in rows], dtype=torch.int64, device="cuda")


def prepare(case, seed):
    return {"plan": _prepare_plan, "rope": _prepare_rope, "attn": _prepare_attn, "accept": _prepare_accept}[case["kind"]](case, seed)


def _prepare_plan(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    cs, ts = _lengths(c)
    n, P = len(cs), c["page"]
    need = _pages(c)
    held = [-(-x // P) for x in cs]
    width = max(need) + 3
    total = sum(need) + 7
    ids = torch.randperm(total, device="cuda", generator=g).to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    h = _i32(held).long()
    col = torch.arange(width, device="cuda")
    table = torch.where(col < h[:, None], ids[((torch.cumsum(h, 0) - h)[:, None] + col).clamp(max=total - 1)], table)
    tokens = sum(ts)
    s = dict(case=c, page=P, tokens=tokens, ctx=_i32(cs), new=_i32(ts), held=_i32(held), table=table,
             free=ids[int(sum(held)):].contiguous(), parents=None, words=0)
    s["n_free"] = _i32([s["free"].numel()])
    if c["tree"]:
        s["parents"] = _i32(_parents(ts, seed))
        s["words"] = -(-max(ts) // 64)
    e = lambda *shape, dt=torch.int32: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
    s.update(table_out=table.clone(), held_out=e(n), n_free_out=e(1), start=e(n + 1), seq=e(n), positions=e(tokens),
             slots=e(tokens), status=e(n), mask=e(tokens, s["words"], dt=torch.int64) if c["tree"] else None)
    if own:
        s["ws"] = torch.empty(_sp().sp_cache_plan_workspace_bytes(n), dtype=torch.uint8, device="cuda")
    return s


def _prepare_rope(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, hq, hk, d = c["tokens"], c["q_heads"], c["kv_heads"], c["head_dim"]
    qkv = torch.randn((t, (hq + 2 * hk) * d), device="cuda", generator=g).mul_(1.5).to(torch.bfloat16)
    q, k, v = (x.view(t, -1, d) for x in qkv.split([hq * d, hk * d, hk * d], 1))
    pages = -(-t // c["page"]) + 2
    cache = [torch.zeros((pages, c["page"], hk, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    order = torch.randperm(pages, device="cuda", generator=g)
    at = torch.arange(t, device="cuda")
    s = dict(case=c, q=q, k=k, v=v, k_cache=cache[0], v_cache=cache[1],
             slots=(order[at // c["page"]] * c["page"] + at % c["page"]).to(torch.int32),
             positions=(at if not c["far"] else torch.randint(0, c["far"], (t,), device="cuda", generator=g)).to(torch.int32),
             q_out=torch.zeros((t, hq, d), dtype=torch.bfloat16, device="cuda"),
             k_out=torch.zeros((t, hk, d), dtype=torch.bfloat16, device="cuda"), qw=None, kw=None, inv_freq=None, eps=1e-6)
    if c["norm"]:
        s["qw"], s["kw"] = (torch.rand((d,), device="cuda", generator=g).add_(0.5).to(torch.bfloat16) for _ in range(2))
    if c["rotary"]:
        r = c["rotary"]
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)).float()
    if own:
        sp = _sp()
        s["shape"] = sp.rope_shape_of(q, k, v, s["q_out"], s["k_out"], c["rotary"], c["interleaved"], s["eps"])
        s["cache"] = sp.cache_shape_of(cache[0])
    return s


def _cache_of(pages, c, g):
    """Keys with a common part (which a sink or the rotation's slow dimensions give) and values of a mean of their own."""
    shape = (pages, c["page"], c["kv_heads"], c["head_dim"])
    k = torch.randn(shape, device="cuda", generator=g, dtype=torch.bfloat16)
    v = torch.randn(shape, device="cuda", generator=g, dtype=torch.bfloat16)
    return k, v


def _prepare_attn(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    cs, ts = _lengths(c)
    n, hq, d = len(cs), c["q_heads"], c["head_dim"]
    need = _pages(c)
    pages = sum(need) + 1
    k, v = _cache_of(pages, c, g)
    ids = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    width = max(need) + 1
    h = _i32(need).long()
    col = torch.arange(width, device="cuda")
    table = torch.where(col < h[:, None], ids[((torch.cumsum(h, 0) - h)[:, None] + col).clamp(max=pages - 1)],
                        torch.full((), -1, dtype=torch.int32, device="cuda"))
    tokens, top = sum(ts), max(ts)
    # queries that look along some keys: logits of a few units, some rows sharp and some flat
    q = torch.randn((tokens, hq, d), device="cuda", generator=g)
    q = (q * (0.5 + 2 * torch.rand((tokens, hq, 1), device="cuda", generator=g))).to(torch.bfloat16)
    start = [0]
    for t in ts:
        start.append(start[-1] + t)
    words = -(-top // 64)
    s = dict(case=c, q=q, k_cache=k, v_cache=v, table=table, seq=_i32([x + y for x, y in zip(cs, ts)]), start=_i32(start),
             mask=_ancestor_words(_parents(ts, seed), ts, words) if top > 1 else None, words=words, top=top,
             longest=max(x + y for x, y in zip(cs, ts)), o=torch.zeros_like(q),
             lse=torch.zeros((tokens, hq), dtype=torch.float32, device="cuda"))
    if own:
        sp = _sp()
        s["cache"] = sp.cache_shape_of(k)
        s["shape"] = sp.step_shape_of(q, s["o"], table, top, words if s["mask"] is not None else 0)
        s["ws"] = torch.empty(sp.sp_cache_attn_workspace_bytes(s["shape"], s["cache"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_accept(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = random.Random(seed)
    cs, ts = _lengths(c)
    n = len(cs)
    need = _pages(c)
    pages = sum(need) + 1
    shape = (c["layers"], pages, c["page"], c["kv_heads"], c["head_dim"])
    k = torch.randn(shape, device="cuda", generator=g, dtype=torch.bfloat16)
    v = torch.randn(shape, device="cuda", generator=g, dtype=torch.bfloat16)
    ids = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    width = max(need) + 1
    h = _i32(need).long()
    col = torch.arange(width, device="cuda")
    table = torch.where(col < h[:, None], ids[((torch.cumsum(h, 0) - h)[:, None] + col).clamp(max=pages - 1)],
                        torch.full((), -1, dtype=torch.int32, device="cuda"))
    paths, counts = [], []
    for t in ts:
        a = min(c["accept"], t)
        # the first tokens of the path lie where they stay; below them it runs through the wide levels of the tree, which come
        # after every place that is written, so that the call can be made again on its own result
        keep = r.randint(0, a)
        keep = a if t - a < a - keep else keep
        p = list(range(keep)) + sorted(r.sample(range(a, t), a - keep))
        counts.append(a)
        paths.append(p + [-1] * (c["accept"] - a))
    return dict(case=c, k_cache=k, v_cache=v, table=table, ctx=_i32(cs), seq=_i32([x + y for x, y in zip(cs, ts)]),
                path=_i32(paths), count=_i32(counts), ctx_out=torch.zeros(n, dtype=torch.int32, device="cuda"),
                cache=_sp().cache_shape_of(k[0]) if own else None)


# ------------------------------------------------------------------------------------------------------------------- runs
def run(s):
    return {"plan": _run_plan, "rope": _run_rope, "attn": _run_attn, "accept": _run_accept}[s["case"]["kind"]](s)


def _run_plan(s):
    out = lambda: {k: s[k] for k in ("table_out", "held_out", "n_free_out", "start", "seq", "positions", "slots", "status",  # noqa: E731
                                     "mask")}
    if own:
        _sp().sp_cache_plan(s["ctx"], s["new"], s["held"], s["table_out"], s["free"], s["n_free"], s["page"], s["parents"],
                            s["held_out"], s["n_free_out"], s["start"], s["seq"], s["positions"], s["slots"], s["status"],
                            s["mask"], s["ws"])
        return out()
    P, ctx, new, held, table = s["page"], s["ctx"].long(), s["new"].long(), s["held"].long(), s["table_out"].long()
    n, width = table.shape
    tokens, words = s["tokens"], s["words"]
    bad = (new < 0) | (ctx < 0) | (held < 0) | (held > width) | (held * P < ctx)
    t = new.clamp(min=0)
    end = t.cumsum(0)
    long = (ctx + new > width * P) | (new > 64 * words if words else new < 0)
    room = end > tokens
    lengths_ok = ~(bad | long | room)
    take = torch.where(lengths_ok, ((ctx + t + P - 1) // P - held).clamp(min=0), 0)
    last = take.cumsum(0)
    n_free = s["n_free"].long().clamp(min=0)
    pages_ok = (take == 0) | (last <= n_free)
    ok = lengths_ok & pages_ok
    status = torch.where(bad, 1, torch.where(long, 2, torch.where(room, 3, torch.where(pages_ok, 0, 4))))
    first = last - take
    col = torch.arange(width, device="cuda")
    fresh = ok[:, None] & (col >= held[:, None]) & (col < (held + take)[:, None])
    free = s["free"].long()
    pick = free[(n_free - 1 - first[:, None] - (col - held[:, None])).clamp(0, free.numel() - 1)]
    table = torch.where(fresh, pick, table)
    start = torch.cat([torch.zeros_like(end[:1]), end.clamp(max=tokens)])
    at = torch.arange(tokens, device="cuda")
    req = torch.searchsorted(start[1:], at, right=True).clamp(max=n - 1)
    i = at - start[req]
    live = (at < start[n]) & ok[req]
    pos = ctx[req] + i
    slots = torch.where(live, table[req, (pos // P).clamp(0, width - 1)] * P + pos % P, -1)
    mask = None
    if words:
        T = 64 * words
        idx = (start[:-1, None] + torch.arange(T, device="cuda")).clamp(max=tokens - 1)
        own_index = torch.arange(T, device="cuda")
        par = s["parents"].long()[idx]
        par = torch.where((par >= 0) & (par < own_index), par, -1)
        step = (par[:, :, None] == own_index).float() + torch.eye(T, device="cuda")
        for _ in range(max(1, (T - 1).bit_length())):
            step = (step @ step).clamp_(max=1)
        anc = step > 0
        pos = ctx[req] + anc[req, i.clamp(max=T - 1)].sum(1) - 1
        row = anc.view(n, T, words, 64).long() << torch.arange(64, device="cuda")
        mask = torch.where(live[:, None], row.sum(3)[req, i.clamp(max=T - 1)], 0)
    positions = torch.where(live, pos, 0)
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return dict(table_out=i32(table), held_out=i32(torch.where(ok, held + take, held)),
                n_free_out=i32(n_free - torch.where(ok, take, 0).sum()), start=i32(start), seq=i32(torch.where(ok, ctx + new, 0)),
                positions=i32(positions), slots=i32(slots), status=i32(status), mask=mask)


def _rotated(x, s, weight):
    c, y = s["case"], x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(2, keepdim=True) + s["eps"]) * weight.float()
    r = c["rotary"]
    if not r:
        return y.to(torch.bfloat16)
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
    a, b = a * cos - b * sin, a * sin + b * cos
    rot = torch.stack([a, b], 3).flatten(2) if c["interleaved"] else torch.cat([a, b], 2)
    return torch.cat([rot, y[..., r:]], 2).to(torch.bfloat16)


def _run_rope(s):
    if own:
        _sp().sp_qk_norm_rope(s["shape"], s["q"], s["k"], s["v"], s["qw"], s["kw"], s["inv_freq"], s["positions"], s["q_out"],
                              s["k_out"], s["cache"], s["k_cache"], s["v_cache"], s["slots"])
    else:
        s["q_out"] = _rotated(s["q"], s, s["qw"])
        s["k_out"] = _rotated(s["k"], s, s["kw"])
        at = s["slots"].long()
        s["k_cache"].view(-1, *s["k"].shape[1:])[at] = s["k_out"]
        s["v_cache"].view(-1, *s["v"].shape[1:])[at] = s["v"]
    return {k: s[k] for k in ("q_out", "k_out", "k_cache", "v_cache")}


def _run_attn(s):
    c = s["case"]
    if own:
        _sp().sp_cache_attn(s["shape"], s["cache"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["seq"], s["start"],
                            s["mask"], s["o"], s["lse"], s["ws"])
        return {"o": s["o"], "lse": s["lse"]}
    P, hq, hk, d, T = c["page"], c["q_heads"], c["kv_heads"], c["head_dim"], s["top"]
    n, g, used = s["table"].shape[0], hq // hk, -(-s["longest"] // P)
    pages = s["table"][:, :used].long().clamp(min=0)
    k, v = (x[pages].view(n, used * P, hk, d).permute(0, 2, 1, 3).float() for x in (s["k_cache"], s["v_cache"]))
    start = s["start"].long()
    idx = (start[:-1, None] + torch.arange(T, device="cuda")).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][idx].float().view(n, T, hk, g, d).permute(0, 2, 1, 3, 4).reshape(n, hk, T * g, d)
    x = (q @ k.transpose(2, 3)).view(n, hk, T, g, -1).mul_(1 / math.sqrt(d))
    ctx = s["seq"].long() - (start[1:] - start[:-1])
    j = torch.arange(used * P, device="cuda") - ctx[:, None]
    if s["mask"] is None:
        seen = (j <= 0)[:, None]
    else:
        word = s["mask"][idx].gather(2, (j // 64).clamp(0, s["words"] - 1)[:, None].expand(-1, T, -1))
        seen = (j < 0)[:, None] | ((j >= 0) & (j < 64 * s["words"]))[:, None] & ((word >> (j.clamp(min=0) % 64)[:, None]) & 1).bool()
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = x.max(4, keepdim=True).values
    p = x.sub_(top).exp_()
    total = p.sum(4, keepdim=True)
    o = (p.view(n, hk, T * g, -1) @ v).view(n, hk, T, g, d) / total
    lse = (top + total.log())[..., 0]
    at = torch.arange(s["q"].shape[0], device="cuda")
    req = torch.searchsorted(start[1:], at, right=True)
    i = at - start[req]
    return {"o": o.permute(0, 2, 1, 3, 4)[req, i].reshape(-1, hq, d).to(torch.bfloat16),
            "lse": lse.permute(0, 2, 1, 3)[req, i].reshape(-1, hq)}


def _run_accept(s):
    c = s["case"]
    if own:
        _sp().sp_cache_accept(s["cache"], s["k_cache"], s["v_cache"], s["table"], s["ctx"], s["seq"], s["path"], s["count"],
                              s["ctx_out"])
        return {k: s[k] for k in ("k_cache", "v_cache", "ctx_out")}
    P, a = c["page"], c["accept"]
    ctx, path, seq = s["ctx"].long(), s["path"].long(), s["seq"].long()
    order = torch.arange(a, device="cuda")
    before = torch.cat([torch.full_like(path[:, :1], -1), path[:, :-1]], 1)
    fine = (order < s["count"].long()[:, None]) & (path > before) & (path < (seq - ctx)[:, None])
    fine = fine.long().cumprod(1).bool()
    row = torch.arange(ctx.numel(), device="cuda")[:, None]
    table = s["table"].long()

    def slot(pos):
        return table[row, (pos // P).clamp(max=table.shape[1] - 1)] * P + pos % P

    # behind the path's end the first move is made again
    to = slot(ctx[:, None] + torch.where(fine, order, 0))
    source = slot(ctx[:, None] + torch.where(fine, path, path[:, :1]))
    s["ctx_out"] = (ctx + fine.sum(1)).to(torch.int32)
    for x in (s["k_cache"], s["v_cache"]):
        flat = x.view(c["layers"], -1, c["kv_heads"], c["head_dim"])
        flat[:, to.reshape(-1)] = flat[:, source.reshape(-1)]
    return {k: s[k] for k in ("k_cache", "v_cache", "ctx_out")}


# ------------------------------------------------------------------------------------------------------------------- work
def work(case):
    """Bytes: each input once and each output once.  Operations: products and sums of the definition."""
    c = case
    if c["kind"] == "rope":
        row = c["head_dim"] * 2 * c["tokens"]
        read = (c["q_heads"] + 2 * c["kv_heads"]) * row + 8 * c["tokens"]
        written = (c["q_heads"] + 3 * c["kv_heads"]) * row
        return {"bytes": read + written, "flops": 7 * (c["q_heads"] + c["kv_heads"]) * c["head_dim"] * c["tokens"]}
    cs, ts = _lengths(c)
    n, tokens = len(cs), sum(ts)
    if c["kind"] == "plan":
        fresh = sum(max(0, -(-(x + y) // c["page"]) + -x // c["page"]) for x, y in zip(cs, ts))
        per_token = 8 + (4 + 8 * (-(-max(ts) // 64)) if c["tree"] else 0)
        return {"bytes": n * 28 + fresh * 8 + tokens * per_token, "flops": 0}
    if c["kind"] == "attn":
        kv = sum(x + y for x, y in zip(cs, ts)) * c["kv_heads"] * c["head_dim"] * 4
        pairs = sum((x + y) * y for x, y in zip(cs, ts))
        return {"bytes": kv + tokens * c["q_heads"] * (c["head_dim"] * 4 + 4), "flops": 4 * pairs * c["q_heads"] * c["head_dim"]}
    moved = sum(min(c["accept"], t) for t in ts)
    return {"bytes": moved * c["layers"] * c["kv_heads"] * c["head_dim"] * 8 + n * 16, "flops": 0}


# ------------------------------------------------------------------------------------------------------------------ exact
def exact(case, seed):
    return {"plan": _exact_plan, "rope": _exact_rope, "attn": _exact_attn, "accept": _exact_accept}[case["kind"]](case, seed)


def _exact_plan(c, seed):
    """Request by request, token by token, as the plan is defined."""
    s = _prepare_plan(c, seed)
    ctx, new, held, free = (s[k].tolist() for k in ("ctx", "new", "held", "free"))
    table, n_free = s["table"].tolist(), int(s["n_free"])
    parents, P = None if s["parents"] is None else s["parents"].tolist(), s["page"]
    start, seq, positions, slots, masks = [0], [], [], [], []
    for r in range(len(ctx)):
        while held[r] * P < ctx[r] + new[r]:
            n_free -= 1
            table[r][held[r]] = free[n_free]
            held[r] += 1
        seq.append(ctx[r] + new[r])
        up, deep = [], []
        for i in range(new[r]):
            p = ctx[r] + i
            slots.append(table[r][p // P] * P + p % P)
            if parents is None:
                positions.append(p)
                continue
            q = parents[start[-1] + i]
            up.append((1 << i) | (up[q] if q >= 0 else 0))
            deep.append(deep[q] + 1 if q >= 0 else 0)
            positions.append(ctx[r] + deep[i])
        masks += up
        start.append(start[-1] + new[r])
    mask = None
    if parents is not None:
        m = [[(x >> (64 * w)) & ((1 << 64) - 1) for w in range(s["words"])] for x in masks]
        mask = torch.tensor([[x - (1 << 64) if x >> 63 else x for x in y] for y in m], dtype=torch.int64)
    t = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return dict(table_out=t(table), held_out=t(held), n_free_out=t([n_free]), start=t(start), seq=t(seq), positions=t(positions),
                slots=t(slots), status=t([0] * len(ctx)), mask=mask)


def _exact_rope(c, seed):
    s = _prepare_rope(c, seed)
    d, r = c["head_dim"], c["rotary"]

    def turned(x, w):
        x = x.double().clone()
        if w is not None:
            x *= w.double() / torch.sqrt(x.square().sum(-1, keepdim=True) / d + s["eps"])
        if r:
            z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double().outer(s["inv_freq"].double()))
            even = torch.arange(0, r, 2, device="cuda") if c["interleaved"] else torch.arange(r // 2, device="cuda")
            odd = even + (1 if c["interleaved"] else r // 2)
            y = torch.complex(x[:, :, even], x[:, :, odd]) * z[:, None]
            x[:, :, even], x[:, :, odd] = y.real, y.imag
        return x

    q, k = turned(s["q"], s["qw"]), turned(s["k"], s["kw"])
    caches = []
    for x in (k, s["v"].double()):
        flat = torch.zeros((s["k_cache"].shape[0] * c["page"],) + tuple(x.shape[1:]), dtype=torch.float64, device="cuda")
        flat.index_copy_(0, s["slots"].long(), x)
        caches.append(flat.view(s["k_cache"].shape))
    return {"q_out": q, "k_out": k, "k_cache": caches[0], "v_cache": caches[1]}


def _exact_attn(c, seed):
    """Request by request and KV head by KV head; a query's keys are the context and its ancestors."""
    s = _prepare_attn(c, seed)
    P, d, g = c["page"], c["head_dim"], c["q_heads"] // c["kv_heads"]
    start, seq = s["start"].tolist(), s["seq"].tolist()
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for r, length in enumerate(seq):
        a, b = start[r], start[r + 1]
        t = b - a
        pages = s["table"][r, :-(-length // P)].long()
        visible = torch.ones((t, length), dtype=torch.bool, device="cuda")
        if s["mask"] is not None:
            bit = torch.arange(t, device="cuda")
            visible[:, length - t:] = ((s["mask"][a:b][:, bit // 64] >> (bit % 64)) & 1) != 0
        bias = torch.zeros((t, 1, length), dtype=torch.float64, device="cuda").masked_fill_(~visible[:, None], -math.inf)
        for h in range(c["kv_heads"]):
            k = s["k_cache"][pages, :, h].reshape(-1, d)[:length].double()
            v = s["v_cache"][pages, :, h].reshape(-1, d)[:length].double()
            q = s["q"][a:b, h * g:(h + 1) * g].double()
            x = (q.reshape(-1, d) @ k.T).view(t, g, length) / math.sqrt(d) + bias
            z = torch.logsumexp(x, 2)
            o[a:b, h * g:(h + 1) * g] = ((x - z[..., None]).exp().view(-1, length) @ v).view(t, g, d)
            lse[a:b, h * g:(h + 1) * g] = z
    return {"o": o, "lse": lse}


def _exact_accept(c, seed):
    s = _prepare_accept(c, seed)
    P = c["page"]
    k, v, table = s["k_cache"].clone(), s["v_cache"].clone(), s["table"].tolist()
    ctx, path, count = s["ctx"].tolist(), s["path"].tolist(), s["count"].tolist()
    where = lambda r, pos: (table[r][pos // P], pos % P)  # noqa: E731
    for r in range(len(ctx)):
        for i in range(count[r]):
            (a, b), (x, y) = where(r, ctx[r] + i), where(r, ctx[r] + path[r][i])
            for cache in (k, v):
                cache[:, a, b] = cache[:, x, y]
    return {"k_cache": k, "v_cache": v, "ctx_out": torch.tensor([a + b for a, b in zip(ctx, count)], dtype=torch.int32)}
