"""Block tables and slot maps from request lengths, against the rules applied sequence by sequence: whole numbers, equal."""
import numpy as np
import pytest
import torch

import cache_ops as R

pytestmark = pytest.mark.gpu


def _case(n, width, bs, seed, most_new, ahead=0):
    rng = np.random.default_rng(seed)
    ctx = rng.integers(0, width * bs + 1, n).astype(np.int32)
    new = np.minimum(rng.integers(0, most_new + 1, n), width * bs - ctx).astype(np.int32)
    held = np.minimum(-(-ctx // bs) + rng.integers(0, ahead + 1, n), width).astype(np.int32)
    ids = rng.permutation(int(held.sum()) + 4 * n * (most_new // bs + 2)).astype(np.int32)
    tables = np.full((n, width), -5, dtype=np.int32)
    at = 0
    for i in range(n):
        tables[i, :held[i]] = ids[at:at + held[i]]
        at += held[i]
    return tables, ctx, new, held, ids[at:]


def _check(tables, ctx, new, held, free, bs, max_rows, use_held=True, stream=None):
    import paper_2503_13773_amd as K
    dev = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (tables, ctx, new, free, held)]
    torch.cuda.synchronize()
    u = K.block_tables_extend(*dev[:4], bs, max_rows=max_rows, held_blocks=dev[4] if use_held else None, stream=stream)
    torch.cuda.synchronize()
    want = R.extend(tables, ctx, new, held if use_held else -(-ctx // bs), free, bs, max_rows)
    got = (dev[0], u.q_start, u.context_lens, u.held_blocks, u.taken[0], u.slot_map, u.positions, u.row_seqs)
    for name, g, w in zip(("tables", "q_start", "context_lens", "held", "taken", "slots", "positions", "seqs"), got, want):
        assert np.array_equal(g.cpu().numpy().astype(np.int64), np.asarray(w).astype(np.int64)), name
    return want


@pytest.mark.parametrize("n,width,bs,most_new", [(1, 1, 1, 1), (1, 40, 16, 500), (3, 7, 4, 1), (64, 256, 16, 1), (255, 9, 8, 30), (256, 9, 8, 30),
                                                  (257, 33, 2, 40), (1024, 5, 32, 3), (1025, 6, 64, 100), (2048, 4, 16, 20), (2049, 4, 16, 20), (4096, 4, 16, 20),
                                                  (9000, 3, 1, 2), (37, 3, 256, 700)])
@pytest.mark.parametrize("use_held", [True, False])
def test_every_length(n, width, bs, most_new, use_held):
    print(f"[case] tables n={n} width={width} bs={bs} new<={most_new} held={use_held}", flush=True)
    tables, ctx, new, held, free = _case(n, width, bs, 17 + n, most_new, ahead=2)
    _check(tables, ctx, new, held, free, bs, int(new.sum()) + 3, use_held)


@pytest.mark.parametrize("n", [5, 300, 5000])
def test_blocks_or_rows_that_run_out(n):
    """Everybody behind the first who does not fit and needs the same gets nothing; those who need no block go on."""
    tables, ctx, new, held, free = _case(n, 8, 16, n, 60, ahead=1)
    need = np.maximum(0, -(-(ctx + new) // 16) - held)
    for share_blocks, share_rows in ((0.5, 1.0), (1.0, 0.5), (0.3, 0.7), (0.0, 1.0), (1.0, 0.0)):
        print(f"[case] tables n={n} blocks {share_blocks} rows {share_rows}", flush=True)
        want = _check(tables, ctx, new, held, free[:int(share_blocks * need.sum())], 16, int(share_rows * new.sum()))
        assert want[1][-1] < new.sum()


def test_lengths_that_make_no_sense_get_nothing():
    bs, width = 16, 4
    ctx = np.array([10, -1, 64, 65, 60, 0, 20, 5, 2 ** 31 - 1, 30], dtype=np.int32)
    new = np.array([3, 5, 1, 1, 5, -4, 0, 2 ** 31 - 1, 7, 6], dtype=np.int32)
    held = np.array([1, 1, 4, 4, 4, 0, 2, 1, 3, 2], dtype=np.int32)
    tables = np.arange(len(ctx) * width, dtype=np.int32).reshape(-1, width)
    want = _check(tables, ctx, new, held, np.arange(100, 120, dtype=np.int32), bs, 40)
    assert want[1].tolist() == [0, 3, 3, 3, 3, 3, 3, 3, 3, 3, 9]
    held[9], held[0] = 5, -1   # more than the table holds; negative
    assert _check(tables, ctx, new, held, np.arange(100, 120, dtype=np.int32), bs, 40)[1][-1] == 0


@pytest.mark.parametrize("n", [3000, 5000])
def test_sums_beyond_32_bits_do_not_wrap(n):
    """Asked rows add up to more than 2^31 (n = 3000) and 2^32 (n = 5000): everybody behind the first is still refused."""
    bs, width = 256, 4096
    ctx, held, new = np.zeros(n, dtype=np.int32), np.zeros(n, dtype=np.int32), np.full(n, bs * width, dtype=np.int32)
    new[0] = 5
    want = _check(np.full((n, width), -1, dtype=np.int32), ctx, new, held, np.arange(4, dtype=np.int32), bs, 16)
    assert want[1][-1] == 5 and want[4] == 1


def test_a_negative_table_entry_gives_no_slot():
    tables = np.array([[3, -1, 7, -1]], dtype=np.int32)
    want = _check(tables, np.array([14], dtype=np.int32), np.array([40], dtype=np.int32), np.array([3], dtype=np.int32),
                  np.array([9], dtype=np.int32), 16, 50)
    assert (want[5][2:18] == -1).all() and (want[5][:2] >= 0).all() and (want[5][18:40] >= 0).all()


def test_an_empty_batch_and_a_side_stream():
    e = np.zeros(0, dtype=np.int32)
    _check(np.zeros((0, 4), dtype=np.int32), e, e, e, np.arange(3, dtype=np.int32), 16, 9)
    tables, ctx, new, held, free = _case(70, 12, 16, 3, 20)
    _check(tables, ctx, new, held, free, 16, int(new.sum()), stream=torch.cuda.Stream())


def test_outputs_that_overlap_inputs_are_refused():
    import paper_2503_13773_amd as K
    n = 6
    tables, lens, new = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((n, 4), (n,), (n,)))
    free = torch.arange(10, dtype=torch.int32, device="cuda")
    u = K.new_table_update(n, 8)
    for bad in (u._replace(context_lens=lens), u._replace(held_blocks=new), u._replace(positions=u.row_seqs),
                u._replace(taken=free[3:4]), u._replace(q_start=tables.view(-1)[2:2 + n + 1])):
        with pytest.raises(K.KvcError) as e:
            K.block_tables_extend(tables, lens, new, free, 16, out=bad)
        assert e.value.status == -10
