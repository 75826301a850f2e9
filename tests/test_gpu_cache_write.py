"""K and V of many tokens through a slot map, and bounds of the keys of filled blocks: exact, byte for byte."""
import numpy as np
import pytest
import torch

import cache_ops as R

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype,hkv,d,bs,rows", [("bf16", 8, 128, 16, 1), ("bf16", 8, 128, 16, 333), ("bf16", 1, 64, 1, 5), ("bf16", 2, 64, 256, 700),
                                                ("f32", 12, 64, 8, 61), ("f32", 4, 128, 2, 97), ("bf16", 40, 128, 16, 50), ("f32", 33, 128, 4, 19),
                                                ("bf16", 3, 64, 32, 1000), ("f32", 1, 64, 16, 2)])
@pytest.mark.parametrize("fused", [False, True])
def test_rows_land_in_their_slots(dtype, hkv, d, bs, rows, fused):
    import paper_2503_13773_amd as K
    print(f"[case] write {dtype} {hkv} x {d} bs {bs} rows {rows} fused {fused}", flush=True)
    rng = np.random.default_rng(rows * 7 + d)
    pool = rows // bs + 9
    k, v = (_normal(rng, (pool, hkv, bs, d), dtype) for _ in range(2))
    slots = rng.permutation(pool * bs)[:rows].astype(np.int64)
    slots[rng.random(rows) < 0.1] = -1
    for i, bad in enumerate((-2 ** 40, pool * bs, pool * bs + 5, 2 ** 62)):   # none of these is a slot
        if rows > 10 + i:
            slots[3 + 2 * i] = bad
    if fused:  # views into rows [q | k | v] of a projection
        qkv = _normal(rng, (rows, 5 + 2 * hkv, d), dtype)
        kn, vn = qkv[:, 5:5 + hkv], qkv[:, 5 + hkv:]
        on = qkv.cuda()
        dk, dv = on[:, 5:5 + hkv], on[:, 5 + hkv:]
    else:
        kn, vn = (_normal(rng, (rows, hkv, d), dtype) for _ in range(2))
        dk, dv = kn.cuda(), vn.cuda()
    gk, gv = k.cuda(), v.cuda()
    K.kv_cache_write(dk, dv, gk, gv, torch.from_numpy(slots).cuda())
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(gk.cpu().view(bits), R.write(k, kn, slots).view(bits))
    assert torch.equal(gv.cpu().view(bits), R.write(v, vn, slots).view(bits))


def test_any_bits_pass_unchanged_and_no_rows_is_no_work():
    import paper_2503_13773_amd as K
    new = torch.arange(2 * 128, dtype=torch.int16).mul_(257).view(torch.bfloat16).view(1, 2, 128).repeat(3, 1, 1).cuda()   # NaNs among them
    k, v = (torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = torch.tensor([0, 17, 63], device="cuda")
    K.kv_cache_write(new, new, k, v, slots, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    for s in slots.tolist():
        assert torch.equal(k[s // 16, :, s % 16].view(torch.int16), new[0].view(torch.int16))
    before = k.clone()
    K.kv_cache_write(new[:0], new[:0], k, v, slots[:0])
    torch.cuda.synchronize()
    assert torch.equal(k.view(torch.int16), before.view(torch.int16))


def test_what_a_copy_could_not_read_is_refused():
    import paper_2503_13773_amd as K
    k, v = (torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    new, slots = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda"), torch.arange(3, device="cuda")
    for kw in (dict(k_new=new.float()), dict(k_new=new[:2]), dict(slot_map=slots.int()), dict(slot_map=slots[:2]), dict(k_cache=k[:3]),
               dict(k_new=new[:1].expand(3, 2, 128)), dict(k_new=new.transpose(0, 1).contiguous().transpose(0, 1)),
               dict(v_new=torch.zeros((3, 2, 256), dtype=torch.bfloat16, device="cuda")[..., ::2]), dict(k_new=new.cpu()), dict(k_cache=k.cpu())):
        with pytest.raises((ValueError, TypeError)):
            K.kv_cache_write(**{**dict(k_new=new, v_new=new, k_cache=k, v_cache=v, slot_map=slots), **kw})
    odd = torch.zeros(3 * 260 + 4, dtype=torch.bfloat16, device="cuda")
    for off, stride in ((1, 264), (0, 260)):    # a start and rows that are not multiples of 16 bytes
        with pytest.raises(K.KvcError) as e:
            K.kv_cache_write(odd.as_strided((2, 2, 128), (stride, 128, 1), off), new[:2], k, v, slots[:2])
        assert e.value.status == -6


# ---- bounds

def _bounds_case(dtype, hkv, d, bs, ctx, new, seed, special=False):
    import paper_2503_13773_amd as K
    rng = np.random.default_rng(seed)
    ctx, new = np.asarray(ctx, dtype=np.int32), np.asarray(new, dtype=np.int32)
    width = max(1, -(-int(ctx.max(initial=1)) // bs)) + 1
    tables, pool = R.scattered(rng, ctx, bs, width)
    k, before = _normal(rng, (pool, hkv, bs, d), dtype), _normal(rng, (pool, hkv, 2, d), dtype)
    if special:
        flat = k.view(-1)
        at = rng.permutation(flat.numel())[:flat.numel() // 50]
        flat[at[0::3]], flat[at[1::3]], flat[at[2::3]] = float("nan"), float("inf"), float("-inf")
        k[0] = -k[0].abs() - 1
    gb = before.cuda()
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    args = (k.cuda(), gb, torch.from_numpy(tables).cuda(), torch.from_numpy(ctx).cuda())
    if (new == 1).all():
        K.key_bounds_update(*args)
        torch.cuda.synchronize()
        first = gb.cpu()
        gb.copy_(before)
        K.key_bounds_update(*args, torch.from_numpy(starts).cuda(), 1)
        torch.cuda.synchronize()
        assert torch.equal(first.float().nan_to_num(7.5), gb.cpu().float().nan_to_num(7.5))
    else:
        K.key_bounds_update(*args, torch.from_numpy(starts).cuda(), max(0, int(new.max())))
        torch.cuda.synchronize()
    want, got = R.bounds(k, before, tables, ctx, new).float(), gb.cpu().float()
    assert torch.equal(want.isnan(), got.isnan()) and torch.equal(want.nan_to_num(7.5), got.nan_to_num(7.5))


@pytest.mark.parametrize("dtype,hkv,d", [("bf16", 8, 128), ("bf16", 3, 64), ("f32", 5, 64), ("f32", 2, 128), ("bf16", 1, 128)])
@pytest.mark.parametrize("bs", [1, 2, 8, 16, 64, 256])
def test_bounds_of_filled_blocks(dtype, hkv, d, bs):
    print(f"[case] bounds {dtype} {hkv} x {d} bs {bs}", flush=True)
    _bounds_case(dtype, hkv, d, bs, [1, bs, bs + 1, 3 * bs, 2 * bs - 1, 5 * bs, 0], [1] * 7, 3)
    ctx = np.array([4 * bs, 5 * bs + 3, bs - 1 if bs > 1 else 1, 7 * bs, 6 * bs + 1, 2 * bs, 9 * bs])
    _bounds_case(dtype, hkv, d, bs, ctx, np.minimum(ctx, [4 * bs, bs, 9, 2 * bs + 1, 0, 1, 9 * bs]), 4)
    _bounds_case(dtype, hkv, d, bs, ctx, ctx, 5, special=True)


@pytest.mark.parametrize("n", [300, 9000])
def test_bounds_of_a_long_prompt_among_many_decode_steps(n):
    """More blocks than a sequence has workgroups, and more sequences than the launch would have in all."""
    ctx, new = np.full(n, 5), np.ones(n, dtype=np.int64)
    ctx[::3], ctx[7], new[7] = 4, 1500, 1499
    _bounds_case("bf16", 5, 64, 4, ctx, new, 6)


def test_bounds_without_work_and_outside_the_pool():
    import paper_2503_13773_amd as K
    k = torch.randn((4, 2, 16, 64), device="cuda")
    bounds = torch.full((4, 2, 2, 64), 3.0, device="cuda")
    tables = torch.tensor([[9, -1, 2, 3]], dtype=torch.int32, device="cuda")
    K.key_bounds_update(k, bounds, tables, torch.tensor([64], dtype=torch.int32, device="cuda"),
                        torch.tensor([0, 64], dtype=torch.int32, device="cuda"), 64)
    K.key_bounds_update(k, bounds, tables[:0], torch.zeros(0, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert (bounds[:2] == 3.0).all() and torch.equal(bounds[2:, :, 0], k[2:].amin(2)) and torch.equal(bounds[2:, :, 1], k[2:].amax(2))
    for kw in (dict(bounds=bounds[:3]), dict(bounds=bounds.bfloat16()), dict(block_tables=tables.long()), dict(context_lens=tables[0])):
        with pytest.raises((ValueError, TypeError)):
            K.key_bounds_update(**{**dict(k_cache=k, bounds=bounds, block_tables=tables,
                                          context_lens=torch.tensor([64], dtype=torch.int32, device="cuda")), **kw})
    with pytest.raises(K.KvcError):   # several new tokens need q_start
        K.key_bounds_update(k, bounds, tables, torch.tensor([64], dtype=torch.int32, device="cuda"), max_query_len=3)
