"""The operators around the cache's blocks as their formulas say, in 64 bits on the CPU, for the tests of the kernels."""
import math

import numpy as np
import torch


def extend(tables, ctx, new, held, free, bs, max_rows):
    """Sequence by sequence: (tables, q_start, context_lens, held, taken, slots, positions, seqs)."""
    tables = tables.copy()
    n, width = tables.shape
    q_start, ctx2, held2 = [0], ctx.copy(), held.copy()
    slots, positions, seqs = (np.full(max_rows, -1, dtype=np.int64) for _ in range(3))
    asked_blocks = asked_rows = taken = 0
    for i in range(n):
        c, w, h = int(ctx[i]), int(new[i]), int(held[i])
        rows = 0
        if w > 0 and 0 <= c <= width * bs and w <= width * bs - c and 0 <= h <= width:
            need = max(0, -(-(c + w) // bs) - h)
            asked_blocks += need
            asked_rows += w
            if (need == 0 or asked_blocks <= len(free)) and asked_rows <= max_rows:
                tables[i, h:h + need] = free[taken:taken + need]
                taken += need
                rows = w
                ctx2[i], held2[i] = c + w, h + need
                for j in range(w):
                    p, r = c + j, q_start[-1] + j
                    b = int(tables[i, p // bs])
                    slots[r] = b * bs + p % bs if b >= 0 else -1
                    positions[r], seqs[r] = p, i
        q_start.append(q_start[-1] + rows)
    return tables, np.array(q_start), ctx2, held2, taken, slots, positions, seqs


def write(cache, new, slots):
    """cache [blocks][heads][bs][d] (torch, any type) with the rows of `new` in their slots."""
    out, bs = cache.clone(), cache.shape[2]
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < cache.shape[0] * bs:
            out[s // bs, :, s % bs] = new[i]
    return out


def bounds(k, before, tables, ctx, new):
    """Bounds after an update: blocks filled by the last new[n] of ctx[n] tokens."""
    out, bs = before.clone(), k.shape[2]
    for n in range(len(ctx)):
        if new[n] <= 0:
            continue
        for j in range(max(ctx[n] - new[n], 0) // bs, ctx[n] // bs):
            b = int(tables[n, j])
            if 0 <= b < k.shape[0]:
                out[b, :, 0], out[b, :, 1] = k[b].float().amin(1).to(k.dtype), k[b].float().amax(1).to(k.dtype)
    return out


def rows_of(ctx, q_start, total):
    """(sequence, position) of every row, None where it belongs to none; without q_start a decode step."""
    if q_start is None:
        return [(n, int(c) - 1) for n, c in enumerate(ctx)]
    out = [None] * total
    for n in range(len(ctx)):
        for r in range(q_start[n], q_start[n + 1]):
            if 0 <= r < total:
                out[r] = (n, int(ctx[n]) - int(q_start[n + 1]) + r)
    return out


def select(q, bounds_, tables, rows, bs, budget, first, last):
    """int32 [rows][kv heads][budget]; rows that belong to no sequence are -7."""
    hkv, d = bounds_.shape[1], q.shape[2]
    group = q.shape[1] // hkv
    out = np.full((len(rows), hkv, budget), -7, dtype=np.int64)
    for r, where in enumerate(rows):
        if where is None:
            continue
        n, p = where
        nb = p // bs + 1 if p >= 0 else 0
        for h in range(hkv):
            if nb <= budget:
                kept = list(range(nb))
            else:
                ids = torch.from_numpy(np.asarray(tables[n, first:nb - last]).astype(np.int64))
                lo, hi = bounds_[ids, h, 0].double()[:, None], bounds_[ids, h, 1].double()[:, None]
                x = q[r, h * group:(h + 1) * group].double()[None]
                score = torch.where(x >= 0, x * hi, x * lo).sum(2).amax(1)
                finite = torch.isfinite(lo).all(2)[:, 0] & torch.isfinite(hi).all(2)[:, 0] & torch.isfinite(x).all()
                score = torch.where(finite, score, math.inf)
                best = torch.sort(score, descending=True, stable=True).indices[:budget - first - last] + first
                kept = sorted(list(range(first)) + best.tolist() + list(range(nb - last, nb)))
            out[r, h] = kept + [-1] * (budget - len(kept))
    return out


def attend(q, k, v, tables, rows, selected, scale):
    """(out, bound): attention in 64 bits and how far a kernel may be off it, element by element; rows of no sequence are NaN in both.

    The bound: a score is a sum of d products (fp32, any order: d + 2 roundings of at most the sum of the products' sizes), whose error e
    moves every weight by a factor exp(+-e), and with the sum of the weights exp(+-2e); the weights of t tokens and their products with V
    are added in fp32 in any order with the rescaling of a running maximum and a join of parts (another t + 64 roundings), an
    exponential is within 2^-21 and a weight is carried in 16 bits and more (2^-15 for bf16); the output is rounded to its type."""
    d, hkv, bs = q.shape[2], k.shape[1], k.shape[2]
    group = q.shape[1] // hkv
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    bound = torch.full(q.shape, math.nan, dtype=torch.float64)
    half, weight = (2.0 ** -8, 2.0 ** -15) if q.dtype == torch.bfloat16 else (2.0 ** -24, 0.0)
    for r, where in enumerate(rows):
        if where is None:
            continue
        n, p = where
        for h in range(hkv):
            at = [(int(tables[n, b]), s) for b in selected[r, h].tolist() if 0 <= b <= (p // bs if p >= 0 else -1)
                  for s in range(min(bs, p + 1 - b * bs))]
            g = slice(h * group, (h + 1) * group)
            if not at:
                out[r, g] = bound[r, g] = 0.0
                continue
            ids, slots = torch.tensor([a for a, _ in at]), torch.tensor([s for _, s in at])
            keys, values = k[ids, h, slots].double(), v[ids, h, slots].double()
            x = q[r, g].double()
            w = torch.softmax(x @ keys.t() * scale, 1)
            out[r, g] = w @ values
            e = (d + 2) * 2.0 ** -24 * (x.abs() @ keys.abs().t()).max().item() * abs(scale) + 2.0 ** -21
            bound[r, g] = half * (w @ values).abs() + (w @ values.abs()) * (2 * e + weight + (2 * len(at) + 64) * 2.0 ** -24) * (1 + half) + 1e-30
    return out, bound


def scattered(rng, ctx, bs, width, spare=3):
    """Block tables for these lengths over a shuffled pool: (tables, blocks in the pool)."""
    need = [-(-int(c) // bs) for c in ctx]
    pool = sum(need) + spare
    ids = rng.permutation(pool).astype(np.int32)
    tables, at = np.full((len(ctx), width), -1, dtype=np.int32), 0
    for n, m in enumerate(need):
        tables[n, :m] = ids[at:at + m]
        at += m
    return tables, pool


def some_lists(rng, rows, hkv, bs, budget, shuffled):
    """Lists for attention: distinct blocks that the row sees, at random; shuffled ones in any order and with entries that do not count."""
    out = np.full((len(rows), hkv, budget), -1, dtype=np.int32)
    for r, where in enumerate(rows):
        if where is None or where[1] < 0:
            continue
        nb = where[1] // bs + 1
        for h in range(hkv):
            m = int(rng.integers(0 if shuffled else 1, min(budget, nb) + 1))
            kept = rng.permutation(nb)[:m]
            if not shuffled:
                out[r, h, :m] = np.sort(kept)
            else:
                places = rng.permutation(budget)
                out[r, h, places[:m]] = kept
                if budget > m:
                    out[r, h, places[m]] = nb + int(rng.integers(0, 3))  # past the row's own block
    return out
