"""The blocks that each query keeps, against scores in 64 bits from the definition: the same places, in order."""
import numpy as np
import pytest
import torch

import cache_ops as R

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DTYPES[dtype])


def _bounds(rng, pool, hkv, d, dtype):
    mean, spread = _normal(rng, (pool, hkv, d), dtype), _normal(rng, (pool, hkv, d), dtype).abs()
    return torch.stack([mean - spread, mean + spread], 2)


def _check(q, bounds, tables, ctx, starts, bs, budget, first, last, workspace=None, **kw):
    import paper_2503_13773_amd as K
    rows = R.rows_of(ctx, starts, q.shape[0])
    out = torch.full((q.shape[0], bounds.shape[1], budget), -7, dtype=torch.int32, device="cuda")
    K.block_select(q.cuda(), bounds.cuda(), torch.from_numpy(tables).cuda(), torch.from_numpy(np.asarray(ctx, dtype=np.int32)).cuda(), budget,
                   block_size=bs, keep_first=first, keep_last=last, out=out, workspace=workspace,
                   q_start=None if starts is None else torch.from_numpy(np.asarray(starts, dtype=np.int32)).cuda(), **kw)
    torch.cuda.synchronize()
    want = R.select(q, bounds, tables, rows, bs, budget, first, last)
    got = out.cpu().numpy().astype(np.int64)
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
    return got


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 8, 128), ("bf16", 8, 8, 64), ("bf16", 14, 2, 64), ("bf16", 7, 1, 128), ("bf16", 20, 1, 64),
                                            ("f32", 16, 4, 64), ("f32", 4, 4, 128), ("f32", 6, 2, 128), ("f32", 18, 2, 64), ("bf16", 10, 2, 128)])
@pytest.mark.parametrize("bs,budget,first,last", [(16, 8, 1, 2), (1, 33, 0, 1), (8, 1, 0, 1), (4, 5, 4, 1), (256, 3, 1, 1), (32, 300, 1, 1)])
def test_decode_rows(dtype, hq, hkv, d, bs, budget, first, last):
    print(f"[case] select {dtype} {hq}/{hkv} x {d} bs {bs} budget {budget} {first}+{last}", flush=True)
    rng = np.random.default_rng(hq + bs)
    ctx = [0, 1, bs, bs * budget, bs * budget + 1, 40 * bs - 1, 61 * bs + bs // 2 + 1, 17 * bs]
    tables, pool = R.scattered(rng, ctx, bs, 61 + budget)
    _check(_normal(rng, (len(ctx), hq, d), dtype), _bounds(rng, pool, hkv, d, dtype), tables, ctx, None, bs, budget, first, last)


@pytest.mark.parametrize("dtype,hq,hkv,d,bs", [("bf16", 8, 2, 128, 16), ("f32", 8, 2, 64, 8), ("bf16", 3, 3, 64, 32)])
def test_rows_of_chunks(dtype, hq, hkv, d, bs):
    """Every row at its own position; rows in front of and behind the sequences are left as they were."""
    print(f"[case] select rows {dtype} {hq}/{hkv} x {d} bs {bs}", flush=True)
    rng = np.random.default_rng(5)
    ctx = [20 * bs + 3, 9 * bs, 0, 31 * bs, 5]
    starts = np.array([2, 2 + 2 * bs + 1, 2 + 2 * bs + 1, 2 + 2 * bs + 1, 40 + 2 * bs, 45 + 2 * bs])
    tables, pool = R.scattered(rng, ctx, bs, 40)
    total = int(starts[-1]) + 3
    got = _check(_normal(rng, (total, hq, d), dtype), _bounds(rng, pool, hkv, d, dtype), tables, ctx, starts, bs, 6, 1, 2)
    assert (got[:2] == -7).all() and (got[-3:] == -7).all() and (got[2:-3] != -7).any()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("rows,hkv,blocks", [(300, 4, 300), (260, 5, 700), (30, 2, 1500), (40, 2, 400), (20, 2, 2100)])
def test_rows_of_chunks_of_every_number_and_length(dtype, d, rows, hkv, blocks):
    """Few and many rows over short and long tables; zero queries among them, whose scores are all equal, and ones that are not finite."""
    print(f"[case] select chunks {dtype} x {d} rows {rows} x {hkv} blocks {blocks}", flush=True)
    rng = np.random.default_rng(blocks)
    bs = 1 if rows < 100 else 2
    ctx = [blocks * bs - 3, rows + 2 * bs, blocks * bs - 1]
    starts = np.array([1, 1 + rows // 2, 1 + rows // 2 + 5, rows])
    tables, pool = R.scattered(rng, ctx, bs, blocks)
    q, bounds = _normal(rng, (rows, 3 * hkv, d), dtype), _bounds(rng, pool, hkv, d, dtype)
    q[3], q[rows - 2, 1] = 0.0, 0.0
    q[4, 0, 0] = float("inf")
    bounds[tables[2, 40], hkv - 1, 1, 2] = float("nan")
    _check(q, bounds, tables, ctx, starts, bs, 24, 1, 2)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("blocks", [60, 130, 300, 511, 513, 2040, 2051, 17000])
def test_decode_rows_of_every_length(dtype, d, blocks):
    """One share, several, more than one launch, more than a workgroup holds; equal scores and what is not finite in each."""
    print(f"[case] select decode {dtype} x {d} blocks {blocks}", flush=True)
    rng = np.random.default_rng(blocks)
    ctx, pool = [blocks, blocks - 1, blocks // 2 + 20, blocks, blocks], 500
    tables = np.stack([rng.integers(0, pool, blocks) for _ in ctx]).astype(np.int32)   # few blocks, many places: scores tie
    q, bounds = _normal(rng, (5, 6, d), dtype), _bounds(rng, pool, 2, d, dtype)
    q[3] = 0.0
    q[4, 5, 1] = float("nan")
    _check(q, bounds, tables, ctx, None, 1, 20, 2, 1)


def test_small_numbers_keep_their_place():
    """Bounds below the smallest normal number against large queries: products of ordinary size."""
    rng = np.random.default_rng(12)
    bs, nb = 16, 200
    tables = rng.permutation(nb)[None].astype(np.int32)
    for dtype, tiny, large in (("bf16", 2.0 ** -130, 2.0 ** 120), ("f32", 2.0 ** -140, 2.0 ** 120), ("bf16", 2.0 ** -128, 1.0)):
        q = (_normal(rng, (1, 4, 128), "f32") * large).to(DTYPES[dtype])
        bounds = torch.sort(_normal(rng, (nb, 2, 2, 128), "f32") * tiny, dim=2).values.to(DTYPES[dtype])
        _check(q, bounds, tables, [nb * bs], None, bs, 30, 1, 1)
    # what tells the blocks apart is tiny beside what they have in common, in the bounds and in the query
    for first in (True, False):
        q = _normal(rng, (1, 4, 128), "f32")
        bounds = torch.sort(_normal(rng, (nb, 2, 2, 128), "f32"), dim=2).values
        bounds[..., :64] = bounds[:1, ..., :64]
        if first:
            q, bounds = q * 2.0 ** 118, torch.cat([bounds[..., :64] * 2.0 ** -118, bounds[..., 64:] * 2.0 ** -134], -1)
        else:
            q[..., 64:] *= 2.0 ** -135
            bounds[..., 64:] *= 2.0 ** 110
        _check(q, bounds, tables, [nb * bs], None, bs, 30, 1, 1)


@pytest.mark.parametrize("ctx,bs,budget", [(30011, 16, 128), (32768, 8, 500), (70000, 16, 64), (9000, 1, 257)])
def test_long_contexts(ctx, bs, budget):
    print(f"[case] select ctx {ctx} bs {bs} budget {budget}", flush=True)
    rng = np.random.default_rng(ctx)
    lens = [ctx, ctx // 3, ctx - 1]
    width = -(-ctx // bs)
    pool = width + 5
    tables = np.stack([rng.permutation(pool)[:width] for _ in lens]).astype(np.int32)   # blocks shared between rows of the table
    _check(_normal(rng, (3, 4, 64), "bf16"), _bounds(rng, pool, 1, 64, "bf16"), tables, lens, None, bs, budget, 1, 2)


def test_equal_scores_go_to_the_lower_block():
    rng = np.random.default_rng(0)
    bs, nb = 16, 700
    tables = np.zeros((3, nb), dtype=np.int32)                   # every place holds the same block
    tables[1] = rng.integers(0, 3, nb)                           # three kinds of block
    tables[2] = np.arange(nb) % 300                              # zero queries: all scores are zeros of either sign
    q, bounds = _normal(rng, (3, 4, 128), "bf16"), _bounds(rng, 300, 2, 128, "bf16")
    q[2] = torch.where(torch.rand(4, 128) < 0.5, 0.0, -0.0).to(torch.bfloat16)
    for budget in (4, 100, 699):
        got = _check(q, bounds, tables, [nb * bs, nb * bs - 3, nb * bs], None, bs, budget, 1, 2)
        assert got[0, 0].tolist() == list(range(budget - 2)) + [nb - 2, nb - 1]


def test_what_is_not_finite_ranks_first():
    rng = np.random.default_rng(1)
    bs, nb = 16, 90
    tables = np.stack([rng.permutation(nb) for _ in range(4)]).astype(np.int32)
    q, bounds = _normal(rng, (4, 8, 64), "f32"), _bounds(rng, nb, 2, 64, "f32")
    for place, value in ((11, float("nan")), (40, float("inf")), (41, float("-inf"))):
        b = tables[0, place]
        bounds[b, 1, 1 if value != float("-inf") else 0, 5] = value
    bounds[tables[0, 60], 0, :, 9] = float("-inf")               # both bounds
    q[2, 3, 7] = float("inf")                                    # a query of its own group only
    q[3] = float("nan")
    got = _check(q, bounds, tables, [nb * bs] * 4, None, bs, 8, 1, 2)
    assert {11, 40, 41} <= set(got[0, 1].tolist()) and 60 in got[0, 0].tolist()
    assert got[3, 0].tolist() == [0, 1, 2, 3, 4, 5, nb - 2, nb - 1]


def test_extreme_values_do_not_overflow():
    """Products near the top of the type's range and far below: 64 bits hold them all."""
    rng = np.random.default_rng(2)
    bs, nb = 16, 70
    tables = rng.permutation(nb)[None].astype(np.int32)
    for dtype in ("f32", "bf16"):
        q = (_normal(rng, (1, 4, 128), "f32") * 1e38).clamp(-3e38, 3e38).to(DTYPES[dtype])
        b = _bounds(rng, nb, 1, 128, "f32")
        b = torch.sort((b * torch.logspace(-30, 37.5, nb)[:, None, None, None]).clamp(-3e38, 3e38), dim=2).values.to(DTYPES[dtype])
        _check(q, b, tables, [nb * bs], None, bs, 20, 1, 1)


def test_a_bound_on_the_lengths_and_workspaces():
    import paper_2503_13773_amd as K
    rng = np.random.default_rng(3)
    bs, ctx = 16, [800, 33, 640]
    tables, pool = R.scattered(rng, ctx, bs, 400)
    q, bounds = _normal(rng, (3, 8, 64), "bf16"), _bounds(rng, pool, 2, 64, "bf16")
    small = K.new_select_workspace(q.cuda(), bounds.cuda(), torch.from_numpy(tables).cuda(), 9, block_size=bs, max_context_len=800)
    large = K.new_select_workspace(q.cuda(), bounds.cuda(), torch.from_numpy(tables).cuda(), 9, block_size=bs)
    assert small.numel() < large.numel()
    small[4096:].fill_(255)   # behind the counters anything may stand
    large[4096:].fill_(255)
    a = _check(q, bounds, tables, ctx, None, bs, 9, 1, 2, workspace=small, max_context_len=800)
    b = _check(q, bounds, tables, ctx, None, bs, 9, 1, 2, workspace=large)
    assert not small[:4096].any() and not large[:4096].any()
    assert np.array_equal(a, b)
    with pytest.raises(K.KvcError) as e:
        _check(q, bounds, tables, ctx, None, bs, 9, 1, 2, workspace=small)
    assert e.value.status == -5
    # a length past the bound counts as the bound
    _check_at = R.select(q, bounds, tables, [(0, 639), (1, 32), (2, 639)], bs, 9, 1, 2)
    out = K.block_select(q.cuda(), bounds.cuda(), torch.from_numpy(tables).cuda(), torch.tensor(ctx, dtype=torch.int32, device="cuda"), 9,
                         block_size=bs, keep_first=1, keep_last=2, max_context_len=640)
    assert np.array_equal(out.cpu().numpy().astype(np.int64), _check_at)


def test_refusals():
    import paper_2503_13773_amd as K
    q, bounds = torch.zeros((2, 4, 64), device="cuda"), torch.zeros((5, 2, 2, 64), device="cuda")
    tables, lens = torch.zeros((2, 9), dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    ok = dict(q=q, bounds=bounds, block_tables=tables, context_lens=lens, budget=4, block_size=16)
    for kw in (dict(budget=0), dict(keep_last=0), dict(keep_first=4), dict(keep_first=-1), dict(keep_first=2 ** 31 - 1, keep_last=2 ** 31 - 1), dict(block_size=12),
               dict(q=q[:1]), dict(max_context_len=16 * 9 + 1)):
        with pytest.raises((K.KvcError, ValueError)):
            K.block_select(**{**ok, **kw})
    for kw in (dict(q=q.bfloat16()), dict(q=q.half()), dict(bounds=bounds[:, :, :1]), dict(bounds=bounds.cpu()), dict(block_tables=tables.long()),
               dict(context_lens=lens[:1]), dict(q_start=lens), dict(out=torch.zeros((2, 2, 5), dtype=torch.int32, device="cuda")),
               dict(out=torch.zeros((2, 2, 4), dtype=torch.int64, device="cuda")), dict(q=q.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises((ValueError, TypeError)):
            K.block_select(**{**ok, **kw})
