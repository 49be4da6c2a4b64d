"""Plain reference of the calls around the paged key/value cache: numpy, 64 bits, request by request and row by row.

Arrays come and go on the host; bf16 data comes widened to float.  Nothing here shares code with the library.
"""
from __future__ import annotations

import numpy as np

OK, BAD_LENGTH, TOO_LONG, NO_ROOM, NO_PAGES = range(5)


def _lacking(ctx, new, held, page):
    return max(0, -(-(ctx + new) // page) - held)


def plan(ctx_len, new_len, n_held, block_table, free_pages, n_free, page, max_tokens, parents=None, words=0):
    """What sp_cache_plan writes, as a dict; `block_table` is copied."""
    n, width = block_table.shape
    table = block_table.copy()
    n_free = max(0, min(int(n_free), len(free_pages)))
    taken, asked, starved = 0, 0, False
    start, seq, held_out, status = [0], [], [], []
    positions, slots = np.zeros(max_tokens, np.int64), np.full(max_tokens, -1, np.int64)
    mask = [[0] * words for _ in range(max_tokens)]
    end = 0
    for r in range(n):
        ctx, new, held = int(ctx_len[r]), int(new_len[r]), int(n_held[r])
        end += max(new, 0)
        if new < 0 or ctx < 0 or held < 0 or held > width or held * page < ctx:
            st = BAD_LENGTH
        elif ctx + new > width * page or (words and new > 64 * words):
            st = TOO_LONG
        elif end > max_tokens:
            st = NO_ROOM
        else:
            lack = _lacking(ctx, new, held, page)
            asked += lack
            starved = asked > n_free
            st = NO_PAGES if lack and starved else OK
        if st == OK:
            for e in range(held, held + lack):
                table[r, e] = free_pages[n_free - 1 - taken]
                taken += 1
            held += lack
            sees, depth = [], []
            for i in range(new):
                p = i - 1 if parents is None else int(parents[start[-1] + i])
                p = p if 0 <= p < i else -1
                sees.append((1 << i) | (sees[p] if p >= 0 else 0))
                depth.append(depth[p] + 1 if p >= 0 else 0)
                t, pos = start[-1] + i, ctx + i
                slot = int(table[r, pos // page]) * page + pos % page
                slots[t] = slot if 0 <= slot < 2 ** 31 else -1
                positions[t] = ctx + depth[i]
                mask[t] = [(sees[i] >> (64 * w)) & (2 ** 64 - 1) for w in range(words)]
        status.append(st)
        seq.append(ctx + new if st == OK else 0)
        held_out.append(held)
        start.append(min(end, max_tokens))
    return dict(table=table, n_held=np.array(held_out), n_free=n_free - taken, tok_start=np.array(start), seq_len=np.array(seq),
                positions=positions, slots=slots, status=np.array(status),
                mask=np.array(mask, dtype=np.uint64).reshape(max_tokens, words))


def norm_rope(x, weight, eps, positions, inv_freq, rotary, interleaved):
    """x [tokens][heads][d] -> (result, scale of its rounding errors), both 64 bits."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    y, size = x.copy(), np.abs(x)
    if rotary:
        a = np.arange(0, rotary, 2) if interleaved else np.arange(rotary // 2)
        b = a + 1 if interleaved else a + rotary // 2
        # 64-bit products of 32-bit factors; extended precision where the platform has it
        turn = (np.asarray(positions, np.longdouble)[:, None] * np.asarray(inv_freq, np.longdouble)) % (2 * np.longdouble(
            "3.14159265358979323846264338327950288"))
        c, s = np.cos(turn).astype(np.float64)[:, None], np.sin(turn).astype(np.float64)[:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


def attention(q, k_cache, v_cache, block_table, seq_len, tok_start, mask, scale):
    """q [tokens][hq][d], caches [pages][page][hkv][d], mask uint64 [tokens][words] or None (chains).

    Returns o, lse and what bounds their errors: sum p |v| and the largest sum |q k| * scale of a row; rows behind the last
    token are NaN."""
    n_tok, hq, d = q.shape
    n_pages, page, hkv, _ = k_cache.shape
    group, width = hq // hkv, block_table.shape[1]
    o = np.full((n_tok, hq, d), np.nan)
    size = np.full((n_tok, hq, d), np.nan)
    lse, logit = np.full((n_tok, hq), np.nan), np.zeros((n_tok, hq))
    for r in range(len(seq_len)):
        t0, t1 = int(tok_start[r]), int(tok_start[r + 1])
        new, length = t1 - t0, min(int(seq_len[r]), width * page)
        if new <= 0:
            continue
        if length < new:
            length = 0
        ctx = length - new
        pages = np.array([block_table[r, p // page] for p in range(length)], np.int64)
        exists = (pages >= 0) & (pages < n_pages)
        at = np.where(exists, pages, 0), np.arange(length) % page
        k, v = k_cache[at].astype(np.float64), v_cache[at].astype(np.float64)   # [keys][hkv][d]
        for i in range(new):
            sees = exists.copy()
            for j in range(new if length else 0):
                bit = j <= i if mask is None else j < 64 * mask.shape[1] and (int(mask[t0 + i, j // 64]) >> (j % 64)) & 1
                sees[ctx + j] &= bool(bit)
            for h in range(hq):
                ks, vs = k[sees, h // group], v[sees, h // group]
                if not len(ks):
                    o[t0 + i, h], lse[t0 + i, h], size[t0 + i, h] = 0, -np.inf, 0
                    continue
                qr = q[t0 + i, h].astype(np.float64)
                x = ks @ qr * scale
                top = x.max()
                p = np.exp(x - top)
                lse[t0 + i, h] = top + np.log(p.sum())
                p /= p.sum()
                with np.errstate(invalid="ignore"):
                    o[t0 + i, h] = (p[:, None] * vs).sum(0)
                    size[t0 + i, h] = (p[:, None] * np.abs(vs)).sum(0)
                logit[t0 + i, h] = (np.abs(ks) @ np.abs(qr)).max() * scale
    return o, lse, size, logit


def accept(k_cache, v_cache, block_table, ctx_len, seq_len, path, count):
    """Caches [layers][pages][page][..], changed in place; returns the new contexts."""
    n_pages, page = k_cache.shape[1:3]
    out = []

    def place(r, pos):
        e = pos // page
        p = int(block_table[r, e]) if e < block_table.shape[1] else -1
        return (p, pos % page) if 0 <= p < n_pages else None

    for r in range(len(ctx_len)):
        ctx, last, n = int(ctx_len[r]), -1, 0
        for x in path[r][:max(0, int(count[r]))]:
            if ctx < 0 or not last < int(x) < int(seq_len[r]) - ctx:
                break
            last = int(x)
            to, source = place(r, ctx + n), place(r, ctx + last)
            if to and source:
                for c in (k_cache, v_cache):
                    c[(slice(None),) + to] = c[(slice(None),) + source]
            n += 1
        out.append(ctx + n)
    return np.array(out)
