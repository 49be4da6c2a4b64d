"""Attention over long contexts: the paths that short ones never reach.  A wavefront of the tiled kernel takes the pages of 64 steps
of 32 keys at a time, one of the kernel for few rows those of 32 steps, the join 64 chunks; each of them has to go on from there."""
import numpy as np
import pytest

from tests.test_gpu_cache import HALF_BF16, _attend, _step

pytestmark = pytest.mark.gpu


def _reference(s, rows=None):
    """The definition in 64 bits, a request and a KV head at a time; `rows`: tokens to compute (all).  Returns o, lse and what bounds
    their errors: sum p |v| and the largest |q| |k| scale of a row."""
    import torch
    q, k, v = (s[x].cuda() for x in ("q", "k", "v"))
    n_tok, hq, d = q.shape
    n_pages, page, hk, _ = k.shape
    group, scale = hq // hk, s["scale"] or d ** -0.5
    o, size = torch.zeros(n_tok, hq, d, dtype=torch.float64, device="cuda"), torch.zeros(n_tok, hq, d, dtype=torch.float64, device="cuda")
    lse, logit = (torch.zeros(n_tok, hq, dtype=torch.float64, device="cuda") for _ in range(2))
    table = torch.tensor(np.asarray(s["table"]), device="cuda")
    for r in range(len(s["seq"])):
        t0, t1, length = int(s["start"][r]), int(s["start"][r + 1]), int(s["seq"][r])
        new, ctx = t1 - t0, length - (t1 - t0)
        toks = torch.tensor([t for t in range(t0, t1) if rows is None or t in rows], dtype=torch.long, device="cuda")
        if not len(toks):
            continue
        at = torch.arange(length, device="cuda")
        ids = table[r][at // page]
        exists = (ids >= 0) & (ids < n_pages)
        if s["mask"] is None:
            sees = at[None] - ctx <= (toks - t0)[:, None]
        else:
            words = torch.from_numpy(s["mask"].view(np.int64)).cuda()[toks]
            j = (at - ctx).clamp(min=0)
            sees = (at < ctx)[None] | ((words[:, j // 64] >> (j % 64)) & 1).bool()
        sees = sees & exists[None]
        ids = torch.where(exists, ids, 0)
        for h in range(hk):
            ks, vs = k[ids, at % page, h].double(), v[ids, at % page, h].double()
            ks = torch.where(exists[:, None], ks, 0.0)
            kinds = [(vs == float("inf")) & exists[:, None], (vs == -float("inf")) & exists[:, None], vs.isnan() & exists[:, None]]
            vs = torch.where(exists[:, None] & vs.isfinite(), vs, 0.0)
            for g in range(group):
                x = torch.where(sees, (q[toks, h * group + g].double() @ ks.t()) * scale, -float("inf"))
                top = x.max(1).values
                p = torch.where(sees, torch.exp(x - top.clamp(min=-1e300)[:, None]), 0.0)
                total = p.sum(1)
                lse[toks, h * group + g] = top + total.log()
                p = p / total.clamp(min=1e-300)[:, None]
                y = p @ vs
                for kind, value in zip(kinds, (float("inf"), -float("inf"), float("nan"))):
                    if kind.any():
                        y = torch.where(sees.double() @ kind.double() > 0, y + value, y)
                o[toks, h * group + g], size[toks, h * group + g] = y, p @ vs.abs()
                logit[toks, h * group + g] = q[toks, h * group + g].double().norm(dim=1) * ks.norm(dim=1).max() * scale
    return tuple(x.cpu().numpy() for x in (o, lse, size, logit))


def _close(s, got, rows=None):
    """Tolerances: o, the weights' rounding to bf16, half a step each, twice (in the sum and in its normaliser), and the result's:
    3 * 2^-8 of sum p |v|; the logits' 32-bit sums of d products, (d + 8) 2^-24 of |q| |k| each way.  lse: that, the sum's own rounding
    (2^-24 per addition, len / 16 of them in a row), and 2^-20 and 2^-21 of itself for exp and log."""
    d = s["q"].shape[2]
    pick = np.arange(len(s["q"])) if rows is None else np.array(sorted(rows))
    o, lse, size, logit = (x[pick] for x in _reference(s, rows))
    err = (d + 8) * 2.0 ** -24 * logit
    with np.errstate(invalid="ignore"):
        near = np.abs(o - got[0][pick]) <= 1.01 * ((3 * HALF_BF16 + 2 * err)[..., None] * size) + 2.0 ** -100
        same = np.where(np.isfinite(o), near, (o == got[0][pick]) | (np.isnan(o) & np.isnan(got[0][pick])))
        assert same.all(), (np.argwhere(~same)[:5], got[0][pick][~same][:5], o[~same][:5])
        tol = err + s["seq"].max() / 16 * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -21 * np.abs(np.where(np.isinf(lse), 0, lse))
        fine = np.where(np.isinf(lse), got[1][pick] == lse, np.abs(got[1][pick] - lse) <= tol)
    assert fine.all(), (np.argwhere(~fine)[:5], got[1][pick][~fine][:5], lse[~fine][:5])


# (rows per KV head, chunk in steps of 32 keys): 160 rows 92 steps; 1024 rows 160; 512 rows 376; 160 rows, d 128, 92
@pytest.mark.parametrize("hq,hk,d,new,ctx,steps", [(8, 1, 64, 20, 50000, 92), (32, 2, 64, 64, 40000, 160), (64, 8, 128, 64, 48000, 376),
                                                   (8, 1, 128, 20, 50000, 92)])
def test_tiles_over_chunks_of_more_than_64_steps(hq, hk, d, new, ctx, steps):
    """Pages that do not exist in the first 64 steps of a chunk, behind them, and behind 128, at places of one 16-key half of a step;
    then an infinite value that every row sees behind 64 steps, which sends the tile through its careful pass."""
    page = 16
    s = _step([ctx, 77], [new, 3], hq, hk, d, page, 1, ctx + new)
    print(f"[long] {hq}/{hk} d{d}, {new} over {ctx}", flush=True)
    _close(s, _attend(s))
    clean = s["table"].copy()
    for holes in ([3], [66], [70, 71], [5, 67], [63, 64, 65], [steps - 1], [steps, steps + 64]):
        s["table"] = clean.copy()
        for n, step in enumerate(holes):                       # one half of the step's keys, or the other
            s["table"][0, 2 * step + n % 2] = -1 if n % 2 else s["k"].shape[0]
        print(f"[long] holes in steps {holes}", flush=True)
        _close(s, _attend(s))
    for step, e in ((2, 5), (65, 3), (steps - 1, d - 1)):
        v = s["v"].clone()
        one = dict(s, table=clean.copy(), v=v)
        v[int(clean[0, 2 * step]), 7, 0, e] = float("inf")
        v[int(clean[0, 2 * step + 1]), 2, hk - 1, e - 1] = float("nan")
        one["table"][0, 2 * 68 + 1] = -1
        print(f"[long] odd values in step {step}", flush=True)
        _close(one, _attend(one))


def test_few_row_kernel_over_more_steps_than_it_keeps_pages_of():
    """A request of far more tokens than max_new says goes through the kernel for few rows with chunks of more than 32 of its steps."""
    s = _step([10500, 3], [512, 1], 16, 16, 64, 16, 0, 3)
    rows = set(range(0, 512, 37)) | {511, 512}
    print("[long] 512 tokens, max_new 1", flush=True)
    got = _attend(s, top=1)
    _close(s, got, rows)
    wide = _attend(s)
    err = 3 * HALF_BF16 * 2 * np.abs(s["v"].float().numpy()).max()
    assert np.abs(got[0] - wide[0]).max() <= err
    s["table"][0, 300:303] = -1                                # in the first chunk, behind 32 steps of 128 keys, and in another
    s["table"][0, 520] = s["k"].shape[0]
    s["table"][0, 601] = -1
    got = _attend(s, top=1)
    _close(s, got, rows)
    v = s["v"].clone()
    v[int(s["table"][0, 290]), 3, :, 9] = float("inf")
    s["v"] = v
    _close(s, _attend(s, top=1), rows)


@pytest.mark.parametrize("d,hq,ctx", [(64, 1, 70000), (128, 4, 131071), (64, 16, 66000)])
def test_more_than_64_chunks(d, hq, ctx):
    """One token: 65 to 128 chunks, joined 64 at a time; the largest score in the first chunk, in the last, and in the 65th."""
    import torch
    s = _step([ctx, 5, 9000], [1, 1, 1], hq, 1, d, 64, 0, ctx)
    print(f"[long] one token over {ctx}", flush=True)
    _close(s, _attend(s))
    k = s["k"].clone()
    for at in (10, ctx - 2, 64 * 1024 + 100):
        s["k"] = k.clone()
        s["k"][int(s["table"][0, at // 64]), at % 64, 0] = 4 * s["q"][0, 0] / s["q"][0, 0].float().norm() * 3
        _close(s, _attend(s))
        v = s["v"]
        s["v"] = v.clone()
        s["v"][int(s["table"][0, (ctx - 900) // 64]), 5, 0, 6] = -float("inf")
        _close(s, _attend(s))
        s["v"] = v


@pytest.mark.parametrize("hq,hk,d,news,ctx", [(4, 1, 64, [700, 1, 333], [0, 40, 1000]), (8, 2, 128, [1000], [3001]), (8, 8, 128, [513, 64], [17, 0]),
                                              (28, 4, 128, [2050], [0]), (4, 4, 64, [4500], [700])])
def test_prompts_behind_a_cached_prefix(hq, hk, d, news, ctx):
    """Chains of hundreds to thousands of tokens, over nothing and over a prefix: every token sees those up to itself."""
    s = _step(ctx, news, hq, hk, d, 32, 0, sum(news))
    total = sum(news)
    rows = set(range(0, total, 61)) | set(range(min(total, 70))) | {total - 1, news[0] - 1, total // 2}
    print(f"[long] prompts of {news} behind {ctx}", flush=True)
    _close(s, _attend(s), rows)
