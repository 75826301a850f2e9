"""Attention over chosen blocks against the formula in 64 bits, with a bound on the error derived element by element."""
import math

import numpy as np
import pytest
import torch

import cache_ops as R

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DTYPES[dtype])


def _check(q, k, v, tables, ctx, starts, selected, scale, **kw):
    import paper_2503_13773_amd as K
    rows = R.rows_of(ctx, starts, q.shape[0])
    out = torch.full(q.shape, math.nan, dtype=q.dtype, device="cuda")
    K.paged_attention_selected(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(tables).cuda(),
                               torch.from_numpy(np.asarray(ctx, dtype=np.int32)).cuda(), torch.from_numpy(selected).cuda(), scale, out=out,
                               q_start=None if starts is None else torch.from_numpy(np.asarray(starts, dtype=np.int32)).cuda(), **kw)
    torch.cuda.synchronize()
    want, bound = R.attend(q, k, v, tables, rows, selected, scale)
    got = out.cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    off = (got - want).abs() - bound
    assert not (off > 0).any(), (off.nan_to_num(-1).max().item(), (got - want).abs().nan_to_num(0).max().item())
    return got


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 8, 128), ("bf16", 8, 2, 64), ("bf16", 5, 5, 64), ("bf16", 14, 2, 128), ("bf16", 16, 1, 64),
                                            ("bf16", 40, 2, 128), ("bf16", 17, 1, 64), ("f32", 16, 4, 64), ("f32", 3, 3, 128), ("f32", 12, 2, 64),
                                            ("f32", 20, 1, 128)])
@pytest.mark.parametrize("bs,budget", [(16, 12), (1, 70), (2, 33), (4, 21), (8, 9), (32, 5), (64, 4), (256, 2)])
@pytest.mark.parametrize("shuffled", [False, True])
def test_decode_rows(dtype, hq, hkv, d, bs, budget, shuffled):
    print(f"[case] selected {dtype} {hq}/{hkv} x {d} bs {bs} budget {budget} shuffled {shuffled}", flush=True)
    rng = np.random.default_rng(hq * 3 + bs)
    ctx = [1, 0, bs, 3 * bs + bs // 2 + 1, 40 * bs, 17 * bs - 1, 29 * bs + 1]
    tables, pool = R.scattered(rng, ctx, bs, 45)
    q, k, v = _normal(rng, (len(ctx), hq, d), dtype), _normal(rng, (pool, hkv, bs, d), dtype), _normal(rng, (pool, hkv, bs, d), dtype)
    selected = R.some_lists(rng, R.rows_of(ctx, None, len(ctx)), hkv, bs, budget, shuffled)
    _check(q, k, v, tables, ctx, None, selected, 1 / math.sqrt(d))


@pytest.mark.parametrize("dtype,hq,hkv,d,bs", [("bf16", 8, 2, 128, 16), ("bf16", 4, 4, 64, 32), ("f32", 6, 2, 64, 8), ("bf16", 6, 2, 64, 4)])
def test_rows_of_chunks(dtype, hq, hkv, d, bs):
    print(f"[case] selected rows {dtype} {hq}/{hkv} x {d} bs {bs}", flush=True)
    rng = np.random.default_rng(6)
    ctx = [20 * bs + 3, 9 * bs, 0, 31 * bs, 5]
    starts = np.array([2, 40, 40, 40, 75, 80])
    tables, pool = R.scattered(rng, ctx, bs, 40)
    q, k, v = _normal(rng, (83, hq, d), dtype), _normal(rng, (pool, hkv, bs, d), dtype), _normal(rng, (pool, hkv, bs, d), dtype)
    for shuffled in (False, True):
        selected = R.some_lists(rng, R.rows_of(ctx, starts, 83), hkv, bs, 9, shuffled)
        got = _check(q, k, v, tables, ctx, starts, selected, 0.11)
        assert got[:2].isnan().all() and got[80:].isnan().all()


@pytest.mark.parametrize("hq,hkv,d,bs", [(16, 8, 64, 32), (24, 8, 128, 16), (8, 8, 64, 4), (20, 4, 64, 8), (40, 2, 128, 4), (8, 8, 64, 256)])
def test_many_rows(hq, hkv, d, bs):
    """Enough rows for a wavefront each; rows of no sequence in front and behind, lists of any order with gaps."""
    print(f"[case] selected many rows {hq}/{hkv} x {d} bs {bs}", flush=True)
    rng = np.random.default_rng(hq + d)
    rows = 2100 // hkv // (-(-hq // hkv // 16)) + 9
    ctx = [7 * bs + 1 + rows // 2, 0, 3 * bs + rows]
    starts = np.array([1, 1 + rows // 2, 1 + rows // 2, rows - 2])
    tables, pool = R.scattered(rng, ctx, bs, 20 + (rows + 8 * bs) // bs)
    q, k, v = _normal(rng, (rows, hq, d), "bf16"), _normal(rng, (pool, hkv, bs, d), "bf16"), _normal(rng, (pool, hkv, bs, d), "bf16")
    for shuffled in (False, True):
        selected = R.some_lists(rng, R.rows_of(ctx, starts, rows), hkv, bs, 7, shuffled)
        selected[5] = -1
        got = _check(q, k, v, tables, ctx, starts, selected, 0.1)
        assert got[0].isnan().all() and got[-2:].isnan().all() and (got[5] == 0).all()


@pytest.mark.parametrize("dtype,hq,hkv,d,rows,ctx,budget,bs", [("bf16", 32, 8, 128, 1, 30011, 128, 16), ("bf16", 64, 8, 128, 5, 9000, 200, 16),
                                                               ("bf16", 12, 12, 64, 3, 12000, 100, 32), ("f32", 16, 4, 64, 2, 9000, 260, 8),
                                                               ("bf16", 4, 1, 128, 1, 20000, 1100, 16), ("bf16", 2, 1, 64, 1, 5000, 700, 4),
                                                               ("f32", 2, 2, 128, 1, 3000, 900, 2)])
def test_long_lists(dtype, hq, hkv, d, rows, ctx, budget, bs):
    print(f"[case] selected long {dtype} {hq}/{hkv} x {d} rows {rows} ctx {ctx} budget {budget} bs {bs}", flush=True)
    rng = np.random.default_rng(ctx)
    lens = [ctx - 7 * i for i in range(rows)]
    width = -(-ctx // bs)
    pool = width + 9
    tables = np.stack([rng.permutation(pool)[:width] for _ in lens]).astype(np.int32)
    q, k, v = _normal(rng, (rows, hq, d), dtype), _normal(rng, (pool, hkv, bs, d), dtype), _normal(rng, (pool, hkv, bs, d), dtype)
    selected = np.stack([np.stack([np.sort(rng.permutation(c // bs)[:budget]) for _ in range(hkv)]) for c in lens]).astype(np.int32)
    selected[:, :, -1] = [[(c - 1) // bs] * hkv for c in lens]
    _check(q, k, v, tables, lens, None, selected, 1 / math.sqrt(d))
    selected[:, 0] = -1                                          # one KV head whose list is empty beside full ones
    selected[:, :, 5:] = -1
    _check(q, k, v, tables, lens, None, selected, 1 / math.sqrt(d))


@pytest.mark.parametrize("dtype,bs", [("bf16", 16), ("bf16", 4), ("bf16", 64), ("f32", 16), ("bf16", 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_nothing_outside_the_list_reaches_the_output(dtype, bs, d):
    """Tokens past the position and blocks that are not chosen hold NaN and infinities."""
    print(f"[case] selected poison {dtype} bs {bs} d {d}", flush=True)
    rng = np.random.default_rng(8)
    ctx = [5 * bs + bs // 2 + 1, 9 * bs + 1, 3]
    tables, pool = R.scattered(rng, ctx, bs, 12)
    q, k, v = _normal(rng, (3, 8, d), dtype), _normal(rng, (pool, 2, bs, d), dtype), _normal(rng, (pool, 2, bs, d), dtype)
    selected = np.full((3, 2, 6), -1, dtype=np.int32)
    for n, c in enumerate(ctx):
        last = (c - 1) // bs
        kept = sorted({0, last} | set(range(1, last, 2)))[:6]
        kept[-1] = last
        selected[n, :, :len(kept)] = kept
        for b in range(last + 1):
            if b not in kept:
                k[tables[n, b]], v[tables[n, b]] = float("nan"), float("inf")
        k[tables[n, last], :, (c - 1) % bs + 1:] = float("nan")
        v[tables[n, last], :, (c - 1) % bs + 1:] = float("-inf")
    _check(q, k, v, tables, ctx, None, selected, 0.2)


@pytest.mark.parametrize("dtype,d,bs", [("bf16", 128, 16), ("bf16", 64, 16), ("f32", 64, 16), ("bf16", 128, 2)])
def test_scores_and_values_that_are_not_finite(dtype, d, bs):
    """As softmax has it: a score of -inf weighs nothing, +inf or NaN makes the row NaN, an infinity in V keeps its sign."""
    import paper_2503_13773_amd as K
    rng = np.random.default_rng(9)
    ctx = [6 * bs] * 5
    tables, pool = R.scattered(rng, ctx, bs, 6)
    q, k, v = _normal(rng, (5, 2, d), dtype), _normal(rng, (pool, 1, bs, d), dtype), _normal(rng, (pool, 1, bs, d), dtype)
    q[:, :, 0] = 1.0
    k[:, :, :, 0] = 0.0
    k[tables[0, 0], 0, :, 0] = float("-inf")                     # a whole first block without a finite score
    k[tables[1, 3], 0, 0, 0] = float("inf")
    k[tables[2, 3], 0, 1, 0] = float("nan")
    v[tables[3, 2], 0, 0, 5] = float("-inf")
    k[tables[4], 0, :, 0] = float("-inf")                        # no finite score at all
    selected = np.tile(np.arange(6, dtype=np.int32), (5, 1, 1))
    out = K.paged_attention_selected(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(tables).cuda(), torch.tensor(ctx, dtype=torch.int32).cuda(),
                                     torch.from_numpy(selected).cuda(), 0.25).float().cpu()
    rows = R.rows_of(ctx, None, 5)
    want, bound = R.attend(q, k.nan_to_num(0.0, 0.0, -1e30), v, tables, rows, selected, 0.25)
    assert ((out[0] - want[0]).abs() <= 1e-2 + 0 * want[0]).all()
    assert out[1].isnan().all() and out[2].isnan().all() and out[4].isnan().all()
    assert (out[3, :, 5] == float("-inf")).all() and out[3, :, :5].isfinite().all() and out[3, :, 6:].isfinite().all()


def test_scales_of_any_sign():
    rng = np.random.default_rng(10)
    ctx = [70, 33]
    tables, pool = R.scattered(rng, ctx, 16, 6)
    for dtype, d in (("bf16", 128), ("bf16", 64), ("f32", 64)):
        q, k, v = _normal(rng, (2, 4, d), dtype), _normal(rng, (pool, 2, 16, d), dtype), _normal(rng, (pool, 2, 16, d), dtype)
        selected = R.some_lists(rng, R.rows_of(ctx, None, 2), 2, 16, 4, False)
        for scale in (0.0, -0.3, 2.0):
            _check(q, k, v, tables, ctx, None, selected, scale)


def test_an_entry_that_appears_twice_counts_twice():
    rng = np.random.default_rng(11)
    tables, pool = R.scattered(rng, [60], 16, 4)
    for dtype, d in (("bf16", 128), ("f32", 64)):
        q, k, v = _normal(rng, (1, 2, d), dtype), _normal(rng, (pool, 2, 16, d), dtype), _normal(rng, (pool, 2, 16, d), dtype)
        _check(q, k, v, tables, [60], None, np.array([[[1, 3, 1], [0, 0, 0]]], dtype=np.int32), 0.1)


def test_refusals():
    import paper_2503_13773_amd as K
    q, k = torch.zeros((2, 4, 64), device="cuda"), torch.zeros((5, 2, 16, 64), device="cuda")
    tables, lens = torch.zeros((2, 9), dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    sel = torch.zeros((2, 2, 3), dtype=torch.int32, device="cuda")
    ok = dict(q=q, k_cache=k, v_cache=k, block_tables=tables, context_lens=lens, selected=sel, scale=0.1)
    for kw in (dict(q=q.bfloat16()), dict(v_cache=k[:4]), dict(selected=sel.long()), dict(selected=sel[:1]), dict(selected=sel[:, :1]), dict(context_lens=lens[:1]),
               dict(out=q.bfloat16()), dict(out=q[:1]), dict(q_start=lens), dict(k_cache=k.cpu()), dict(selected=sel.transpose(0, 1).contiguous().transpose(0, 1)),
               dict(q=q.half(), k_cache=k.half(), v_cache=k.half())):
        with pytest.raises((ValueError, TypeError)):
            K.paged_attention_selected(**{**ok, **kw})
    for kw in (dict(scale=math.inf), dict(scale=math.nan), dict(selected=sel[..., :0]), dict(q=torch.zeros((3, 4, 64), device="cuda"),
               selected=torch.zeros((3, 2, 3), dtype=torch.int32, device="cuda"))):
        with pytest.raises((K.KvcError, ValueError)):
            K.paged_attention_selected(**{**ok, **kw})


def test_a_workspace_of_a_larger_batch_serves_smaller_ones():
    """A batch that needs none itself; smaller ones, whose lists are cut into parts, use what was asked for it."""
    import paper_2503_13773_amd as K
    print("[case] selected workspace of a larger batch", flush=True)
    rng = np.random.default_rng(12)
    hq, hkv, d, bs, budget = 8, 2, 128, 16, 40
    for dtype in ("bf16", "f32"):
        ws = K.new_selected_workspace(torch.zeros((300, hq, d), dtype=DTYPES[dtype], device="cuda"), torch.zeros((9, hkv, bs, d), dtype=DTYPES[dtype], device="cuda"),
                                      torch.zeros((300, 50), dtype=torch.int32, device="cuda"), budget)
        for rows in (300, 150, 65, 9, 1):
            ctx = [int(x) for x in rng.integers(30 * bs, 50 * bs, rows)]
            tables, pool = np.stack([rng.permutation(60)[:50] for _ in ctx]).astype(np.int32), 60
            q, k, v = _normal(rng, (rows, hq, d), dtype), _normal(rng, (pool, hkv, bs, d), dtype), _normal(rng, (pool, hkv, bs, d), dtype)
            selected = R.some_lists(rng, R.rows_of(ctx, None, rows), hkv, bs, budget, False)
            _check(q, k, v, tables, ctx, None, selected, 1 / math.sqrt(d), workspace=ws)
    assert not ws[:4096].any()


@pytest.mark.parametrize("d,bs", [(128, 16), (64, 32), (64, 4)])
def test_decode_rows_on_both_sides_of_the_loads_that_stay(d, bs):
    """Rows of eight units and of more, of up to a device full, in four and eight wavefronts each."""
    rng = np.random.default_rng(13)
    for rows in (4, 5, 20, 40, 70, 129, 160):
        print(f"[case] selected decode rows {rows} x {d} bs {bs}", flush=True)
        ctx = [int(x) for x in rng.integers(0, 40 * bs, rows)]
        tables = np.stack([rng.permutation(60)[:40] for _ in ctx]).astype(np.int32)
        q, k, v = _normal(rng, (rows, 6, d), "bf16"), _normal(rng, (60, 2, bs, d), "bf16"), _normal(rng, (60, 2, bs, d), "bf16")
        selected = R.some_lists(rng, R.rows_of(ctx, None, rows), 2, bs, 19, True)
        _check(q, k, v, tables, ctx, None, selected, 0.1)
