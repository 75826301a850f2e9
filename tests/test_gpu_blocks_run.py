"""The operators around the cache's blocks together, as a serving program calls them: prompts and chunks, then decode steps, eager,
captured and replayed, on a side stream, in the serving loop, and on a pool beyond 4 GiB."""
import math

import numpy as np
import pytest
import torch

import cache_ops as R
import serving_scenario as S
from gpu_util import BF16_TOL

pytestmark = pytest.mark.gpu

HQ, HKV, D, BS, WIDTH, BUDGET = 8, 2, 64, 16, 24, 5
SCALE = 1 / math.sqrt(D)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


class Program:
    """What a program keeps, and its iteration."""

    def __init__(self, n, max_rows, dtype, blocks, seed):
        import paper_2503_13773_amd as K
        self.K, self.n, self.rows, self.dtype = K, n, max_rows, dtype
        gen = torch.Generator().manual_seed(seed)
        self.k = torch.zeros((blocks, HKV, BS, D), dtype=dtype, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.bounds = K.new_key_bounds(self.k)
        self.tables = torch.full((n, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.lens, self.held, self.new = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(3))
        self.free = torch.randperm(blocks, generator=gen).to(torch.int32).cuda()
        self.update = K.new_table_update(n, max_rows)
        self.qkv = torch.zeros((max_rows, HQ + 2 * HKV, D), dtype=dtype, device="cuda")
        self.q = torch.zeros((max_rows, HQ, D), dtype=dtype, device="cuda")
        self.out = torch.zeros_like(self.q)
        self.kept = torch.zeros((max_rows, HKV, BUDGET), dtype=torch.int32, device="cuda")
        a, b = K.new_select_workspace(self.q, self.bounds, self.tables, BUDGET, block_size=BS), K.new_selected_workspace(self.q, self.k, self.tables, BUDGET)
        self.ws = max((x for x in (a, b) if x is not None), key=lambda x: x.numel())   # one serves both

    def iteration(self, stream=None):
        """Writes the new tokens, chooses and attends; the rows behind the last token stay as they are."""
        K, u = self.K, self.update
        K.block_tables_extend(self.tables, self.lens, self.new, self.free, BS, held_blocks=self.held, out=u, stream=stream)
        K.kv_cache_write(self.qkv[:, HQ:HQ + HKV], self.qkv[:, HQ + HKV:], self.k, self.v, u.slot_map, stream=stream)
        K.key_bounds_update(self.k, self.bounds, self.tables, u.context_lens, u.q_start, self.rows, stream=stream)
        K.block_select(self.q, self.bounds, self.tables, u.context_lens, BUDGET, block_size=BS, keep_first=1, keep_last=2, q_start=u.q_start,
                       out=self.kept, workspace=self.ws, stream=stream)
        K.paged_attention_selected(self.q, self.k, self.v, self.tables, u.context_lens, self.kept, SCALE, q_start=u.q_start, out=self.out,
                                   workspace=self.ws, stream=stream)

    def advance(self):
        """What the program takes over between two iterations."""
        taken = int(self.update.taken[0])
        self.lens.copy_(self.update.context_lens)
        self.held.copy_(self.update.held_blocks)
        self.free = self.free.roll(-taken) if taken else self.free   # the front is in use now: it goes to the back
        self.used = getattr(self, "used", 0) + taken


def _feed(p, rng, new):
    rows = int(np.sum(new))
    qkv = torch.from_numpy(rng.standard_normal((p.rows, HQ + 2 * HKV, D)).astype(np.float32)).to(p.dtype)
    p.new.copy_(torch.from_numpy(np.asarray(new, dtype=np.int32)))
    p.qkv.copy_(qkv)
    p.q.copy_(qkv[:, :HQ])
    p.out.fill_(7.0)
    p.kept.fill_(-9)
    return qkv, rows


def _check(p, history, qkv, new, before):
    """history: K and V of every sequence so far, in order (CPU)."""
    at = 0
    rows = []
    for n, m in enumerate(new):
        for j in range(m):
            history[n].append(qkv[at, HQ:])
            rows.append((n, before[n] + j))
            at += 1
    tables, k, v, out, kept = p.tables.cpu().numpy(), p.k.cpu(), p.v.cpu(), p.out.cpu().double(), p.kept.cpu().numpy()
    names = [int(tables[n, b]) for n in range(p.n) for b in range(-(-len(history[n]) // BS))]
    assert len(set(names)) == len(names) and min(names, default=0) >= 0
    for n, h in enumerate(history):   # the cache holds the true tokens
        for j, x in enumerate(h):
            b, s = int(tables[n, j // BS]), j % BS
            assert torch.equal(k[b, :, s], x[:HKV]) and torch.equal(v[b, :, s], x[HKV:]), (n, j)
    bounds = torch.stack([k.float().amin(2), k.float().amax(2)], 2).to(k.dtype)   # of full blocks: all that is read
    padded = rows + [None] * (p.rows - len(rows))
    want = R.select(qkv[:, :HQ], bounds, tables, padded, BS, BUDGET, 1, 2)
    assert np.array_equal(kept[:len(rows)], want[:len(rows)]) and (kept[len(rows):] == -9).all()
    ref, bound = R.attend(qkv[:, :HQ], k, v, tables, padded, kept, SCALE)
    assert ((out - ref).abs()[:len(rows)] <= bound[:len(rows)]).all() and (out[len(rows):] == 7.0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("side", [False, True])
def test_prompts_chunks_and_decode_steps(dtype, side):
    print(f"[case] run {dtype} side stream {side}", flush=True)
    rng, n = np.random.default_rng(1), 4
    p = Program(n, 150, dtype, 80, 2)
    stream = torch.cuda.Stream() if side else None
    history = [[] for _ in range(n)]
    for new in ([70, 0, 33, 1], [10, 100, 16, 15], [1, 1, 1, 1], [0, 47, 60, 1], [1, 1, 1, 0], [1, 1, 1, 1]):
        before = p.lens.tolist()
        qkv, _ = _feed(p, rng, new)
        torch.cuda.synchronize()
        p.iteration(stream)
        torch.cuda.synchronize()
        _check(p, history, qkv, new, before)
        p.advance()


def test_a_captured_iteration_replayed_with_eager_work_between():
    """One graph of an iteration (a padded batch of at most 40 new tokens), replayed for iterations of other lengths and values, an eager iteration
    of another program on the same workspace between the replays."""
    print("[case] run captured", flush=True)
    rng, n = np.random.default_rng(3), 4
    p, other = Program(n, 40, torch.bfloat16, 60, 4), Program(n, 40, torch.bfloat16, 60, 5)
    other.ws = p.ws
    history, others = [[] for _ in range(n)], [[] for _ in range(n)]
    _feed(p, rng, [0] * n)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        p.iteration()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            p.iteration()
    for new in ([20, 0, 13, 1], [1, 1, 1, 1], [3, 30, 0, 7], [1, 1, 1, 1], [1, 0, 1, 1], [0, 0, 0, 0], [40, 0, 0, 0]):
        for prog, hist in ((p, history), (other, others)):
            before, front = prog.lens.tolist(), prog.free
            qkv, _ = _feed(prog, rng, new)
            torch.cuda.synchronize()
            if prog is p:
                graph.replay()
            else:
                prog.iteration()
            torch.cuda.synchronize()
            _check(prog, hist, qkv, new, before)
            prog.advance()
            if prog.free is not front:   # the graph reads the list where it was captured
                front.copy_(prog.free)
                prog.free = front


def test_calls_without_buffers_of_their_own_and_on_a_side_stream_agree():
    import paper_2503_13773_amd as K
    rng = np.random.default_rng(6)
    ctx = [300, 40, 222]
    tables, pool = R.scattered(rng, ctx, BS, WIDTH)
    for dtype in (torch.bfloat16, torch.float32):
        k, v = (torch.from_numpy(rng.standard_normal((pool, HKV, BS, D)).astype(np.float32)).to(dtype).cuda() for _ in range(2))
        q = torch.from_numpy(rng.standard_normal((3, HQ, D)).astype(np.float32)).to(dtype).cuda()
        t, lens, starts = _i32(tables), _i32(ctx), _i32(np.concatenate([[0], np.cumsum(ctx)]))
        seen = []
        torch.cuda.synchronize()
        for stream in (None, torch.cuda.Stream()):
            with torch.cuda.stream(stream) if stream else torch.cuda.stream(torch.cuda.current_stream()):
                bounds = K.new_key_bounds(k)
            K.key_bounds_update(k, bounds, t, lens, starts, max(ctx), stream=stream)
            kept = K.block_select(q, bounds, t, lens, BUDGET, block_size=BS, stream=stream)
            out = K.paged_attention_selected(q, k, v, t, lens, kept, SCALE, stream=stream)
            u = K.block_tables_extend(t.clone() if stream is None else t.clone(), lens, _i32([3, 0, 5]), _i32(np.arange(9) + pool), BS, max_rows=8)
            torch.cuda.synchronize()
            seen.append((bounds, kept, out, u.slot_map))
        assert all(torch.equal(a, b) for a, b in zip(*seen))


def test_the_serving_loop_attends_to_chosen_blocks(oracle_mod):
    """A budget above every table: the same answers as full attention; swapped-in, recomputed and embedded requests included."""
    from paper_2503_13773_amd.serving import HipOps
    ops = HipOps(S.NUM_BLOCKS, S.SWAP_BLOCKS, S.HQ, S.HKV, S.D, S.BS, sparse_budget=S.LMAX)
    srv = S.make_server(ops)
    S.run(srv, oracle_mod, tol=BF16_TOL)
    assert srv.all_done() and srv.stats["swap_ins"] >= 1 and srv.stats["recomputed"] >= 1


@pytest.mark.parametrize("budget,first,last", [(1, 0, 1), (2, 1, 1), (4, 1, 2)])
def test_the_serving_loop_with_a_small_budget_keeps_what_the_definition_keeps(budget, first, last):
    """Each decode call of the loop against the definition on the cache as it is then."""
    from paper_2503_13773_amd.serving import HipOps
    checked = []

    class Ops(HipOps):
        def decode(self, q, tables, lens):
            out = super().decode(q, tables, lens)
            k, v = self.pool[0].cpu(), self.pool[1].cpu()
            rows = [(i, int(c) - 1) for i, c in enumerate(lens)]
            bounds = torch.stack([k.float().amin(2), k.float().amax(2)], 2).to(k.dtype)
            x = torch.from_numpy(np.ascontiguousarray(q).view(np.int16)).view(torch.bfloat16)
            kept = R.select(x, bounds, tables, rows, S.BS, budget, first, last)
            ref, bound = R.attend(x, k, v, tables, rows, kept, S.SCALE)
            assert (torch.from_numpy(out).double() - ref).abs().sub(bound).max() <= 0
            checked.append(int((np.asarray(lens) > budget * S.BS).sum()))
            return out
    srv = S.make_server(Ops(S.NUM_BLOCKS, S.SWAP_BLOCKS, S.HQ, S.HKV, S.D, S.BS, sparse_budget=budget))
    pending = sorted(S.ARRIVALS, key=lambda a: a[1])
    for it in range(400):
        while pending and pending[0][1] <= it:
            rid, _, sp, so, true_out, ttft, tbt = pending.pop(0)
            srv.submit(S.ServedRequest(rid=rid, prompt_len=sp, est_output_len=so, true_output_len=true_out, ttft_slo=ttft, tbt_slo=tbt))
        srv.step()
        if not pending and srv.all_done():
            break
    assert srv.all_done() and sum(checked) > 20


def test_a_pool_beyond_4_gib():
    """Blocks at both ends of caches of 4.9 GB each: offsets pass 32 bits."""
    import paper_2503_13773_amd as K
    print("[case] large pool", flush=True)
    hq, hkv, d, bs, blocks = 32, 8, 128, 16, 150000
    k, v = (torch.empty((blocks, hkv, bs, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bounds = torch.empty((blocks, hkv, 2, d), dtype=torch.bfloat16, device="cuda")
    names = np.array([0, 149999, 131072, 131071, 65536, 149998, 7, 140001], dtype=np.int32)
    n = 8 * bs
    gen = torch.Generator(device="cuda").manual_seed(1)
    kn, vn = (torch.randn((n, hkv, d), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.full((1, 12), -1, dtype=torch.int32, device="cuda")
    u = K.block_tables_extend(table, _i32([0]), _i32([n]), _i32(names), bs, max_rows=n)
    assert u.slot_map.max().item() == 149999 * bs + bs - 1
    K.kv_cache_write(kn, vn, k, v, u.slot_map)
    K.key_bounds_update(k, bounds, table, u.context_lens, u.q_start, n)
    q = torch.randn((1, hq, d), generator=gen, device="cuda", dtype=torch.bfloat16)
    kept = K.block_select(q, bounds, table, u.context_lens, 5, block_size=bs, keep_first=1, keep_last=2)
    out = K.paged_attention_selected(q, k, v, table, u.context_lens, kept, 0.09)
    few = torch.from_numpy(names).long().cuda()
    small = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    kept2 = K.block_select(q, bounds[few].contiguous(), small, u.context_lens, 5, block_size=bs, keep_first=1, keep_last=2)
    out2 = K.paged_attention_selected(q, k[few].contiguous(), v[few].contiguous(), small, u.context_lens, kept2, 0.09)
    torch.cuda.synchronize()
    assert torch.equal(k[few].transpose(1, 2).reshape(n, hkv, d), kn) and torch.equal(v[few].transpose(1, 2).reshape(n, hkv, d), vn)
    assert torch.equal(bounds[few][:, :, 0], k[few].float().amin(2).bfloat16()) and torch.equal(kept, kept2) and torch.equal(out, out2)
