"""The native calls of the operators around the cache's blocks against the general path of the binding: the same bits, the same errors."""
import numpy as np
import pytest
import torch

import cache_ops as R

pytestmark = pytest.mark.gpu


@pytest.fixture
def K(monkeypatch):
    import paper_2503_13773_amd as K
    from paper_2503_13773_amd import binding as B
    counted = {"native": 0}
    native = B._calls()

    class Counting:
        def __getattr__(self, name):
            f = getattr(native, name)

            def call(*a):
                rc = f(*a)
                counted["native"] += rc is not None
                return rc
            return call
    monkeypatch.setattr(B, "_native", Counting())
    return type("K_", (), dict(K.__dict__, counted=counted, general=lambda: monkeypatch.setattr(B, "_on_device", lambda t: False)))


def _inputs(dtype):
    rng = np.random.default_rng(4)
    ctx = [200, 17, 96]
    tables, pool = R.scattered(rng, ctx, 16, 20)
    k, v = (torch.from_numpy(rng.standard_normal((pool, 2, 16, 64)).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    q, new = (torch.from_numpy(rng.standard_normal((3, h, 64)).astype(np.float32)).to(dtype).cuda() for h in (8, 2))
    return k, v, q, new, torch.from_numpy(tables).cuda(), torch.tensor(ctx, dtype=torch.int32, device="cuda")


def _calls(K, dtype, stream):
    k, v, q, new, t, lens = _inputs(dtype)
    bounds, kept, out, u = K.new_key_bounds(k), torch.zeros((3, 2, 5), dtype=torch.int32, device="cuda"), torch.zeros_like(q), K.new_table_update(3, 9)
    a, b = K.new_select_workspace(q, bounds, t, 5, block_size=16), K.new_selected_workspace(q, k, t, 5)
    free, starts = torch.arange(100, 110, dtype=torch.int32, device="cuda"), torch.tensor([0, 200, 217, 313], dtype=torch.int32, device="cuda")
    slots = torch.tensor([5, -1, 40], device="cuda")
    torch.cuda.synchronize()
    K.block_tables_extend(t, lens, torch.full_like(lens, 3), free, 16, out=u, stream=stream)
    K.kv_cache_write(new, new, k, v, slots, stream=stream)
    K.key_bounds_update(k, bounds, t, lens, starts, 200, stream=stream)
    K.block_select(q, bounds, t, lens, 5, block_size=16, out=kept, workspace=a, stream=stream)
    K.paged_attention_selected(q, k, v, t, lens, kept, 0.1, out=out, workspace=b, stream=stream)
    torch.cuda.synchronize()
    return [*u, t, k, v, bounds, kept, out]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("side", [False, True])
def test_both_paths_write_the_same(K, dtype, side):
    stream = torch.cuda.Stream() if side else None
    got = _calls(K, dtype, stream)
    assert K.counted["native"] == 5
    K.general()
    want = _calls(K, dtype, stream)
    assert K.counted["native"] == 5 and all(torch.equal(a, b) for a, b in zip(got, want))


def test_both_paths_raise_the_same(K):
    k, v, q, new, t, lens = _inputs(torch.bfloat16)
    bounds, kept, out = K.new_key_bounds(k), torch.zeros((3, 2, 5), dtype=torch.int32, device="cuda"), torch.zeros_like(q)
    small, free, u = torch.zeros(256, dtype=torch.uint8, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda"), K.new_table_update(3, 9)
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    calls = [lambda: K.block_tables_extend(t, lens, lens, free, 12, out=u), lambda: K.block_tables_extend(t, lens, lens, free, 16, out=u._replace(taken=free[:1])),
             lambda: K.block_tables_extend(t, lens.long(), lens, free, 16, out=u), lambda: K.kv_cache_write(new[:2], new, k, v, slots),
             lambda: K.kv_cache_write(new, new, k, v.cpu(), slots), lambda: K.key_bounds_update(k, bounds, t, lens, max_query_len=2),
             lambda: K.key_bounds_update(k, bounds[:1], t, lens), lambda: K.block_select(q, bounds, t, lens, 5, block_size=16, out=kept, workspace=small),
             lambda: K.block_select(q, bounds, t, lens, 5, block_size=16, out=kept, keep_last=0), lambda: K.block_select(q.half(), bounds, t, lens, 5, block_size=16, out=kept),
             lambda: K.paged_attention_selected(q, k, v, t, lens, kept, float("nan"), out=out), lambda: K.paged_attention_selected(q, k, v, t, lens, kept.long(), 0.1, out=out),
             lambda: K.paged_attention_selected(q, k, v, t, lens, kept, 0.1, out=out[:1])]
    seen = []
    for general in (False, True):
        if general:
            K.general()
        for call in calls:
            with pytest.raises((K.KvcError, ValueError, TypeError)) as e:
                call()
            seen.append((type(e.value), str(e.value)))
    assert seen[:len(calls)] == seen[len(calls):]
