"""What the operators around the cache's blocks refuse before anything is launched, through the C ABI (no GPU)."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE, ALIGN, OVERLAP = 0, -1, -2, -3, -4, -5, -6, -10
P = 1 << 20   # stands for an aligned device address: every call here ends before it is used


@pytest.fixture(scope="module")
def K():
    import paper_2503_13773_amd as K
    if not os.path.exists(K.library_path()):
        from paper_2503_13773_amd.build import build_library
        build_library()
    K.lib()
    return K


def desc(K, **kw):
    d = dict(num_seqs=4, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=16, max_blocks_per_seq=64, num_pool_blocks=100,
             dtype=K.KVC_BF16)
    d.update(kw)
    return K.AttnDesc(**d)


BAD_DESCS = [(dict(num_seqs=-1), SHAPE), (dict(num_q_heads=7), SHAPE), (dict(head_dim=96), UNSUPPORTED), (dict(block_size=12), UNSUPPORTED),
             (dict(block_size=512), UNSUPPORTED), (dict(dtype=5), DTYPE), (dict(max_blocks_per_seq=0), SHAPE), (dict(max_context_len=1025), SHAPE),
             (dict(max_blocks_per_seq=1 << 27), SHAPE), (dict(reserved=1), SHAPE)]


def test_table_update_is_laid_out_as_in_c(tmp_path):
    from paper_2503_13773_amd.binding import TableUpdateArgs
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "kvc.h"\nint main(void) { printf("%zu %zu %zu\\n", '
                   'sizeof(kvc_table_update), offsetof(kvc_table_update, slot_map), offsetof(kvc_table_update, max_rows)); return 0; }')
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")])
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(TableUpdateArgs), TableUpdateArgs.slot_map.offset, TableUpdateArgs.max_rows.offset]


def test_block_tables_extend(K):
    from paper_2503_13773_amd.binding import TableUpdateArgs
    far = [P * (i + 1) for i in range(12)]

    def call(d=None, update=True, tables=far[7], lens=far[8], new=far[9], held=far[10], free=far[11], num_free=10, **kw):
        u = dict(zip(("q_start", "context_lens", "held_blocks", "taken", "slot_map", "positions", "row_seqs"), far), max_rows=32, reserved=0)
        u.update(kw)
        return K.lib().kvc_block_tables_extend(tables, lens, new, held, free, num_free, ctypes.byref(TableUpdateArgs(**u)) if update else None,
                                               ctypes.byref(d or desc(K)), None)
    for kw, status in BAD_DESCS:
        assert call(desc(K, **kw)) == status, kw
    assert call(update=False) == NULL
    for kw in (dict(q_start=None), dict(context_lens=None), dict(slot_map=None), dict(tables=None), dict(lens=None), dict(new=None), dict(free=None)):
        assert call(**kw) == NULL, kw
    for kw in (dict(max_rows=-1), dict(max_rows=2 ** 31 - 1), dict(reserved=1), dict(num_free=-1), dict(num_free=2 ** 31 - 1)):
        assert call(**kw) == SHAPE, kw
    # 4 sequences: outputs of 16 bytes (20, 4, 256, 128) beside one another and the inputs
    for kw in (dict(context_lens=far[8]), dict(held_blocks=far[10] + 12), dict(taken=far[9] + 8), dict(slot_map=far[7] + 4 * 4 * 64 - 8),
               dict(positions=far[4] + 8 * 31), dict(row_seqs=far[5]), dict(q_start=far[1] - 16), dict(tables=far[11] + 36)):
        assert call(**kw) == OVERLAP, kw


def test_kv_cache_write(K):
    def call(d=None, kn=P, vn=2 * P, ks=0, vs=0, kc=3 * P, vc=4 * P, slots=5 * P, rows=6):
        return K.lib().kvc_kv_cache_write(kn, vn, ks, vs, kc, vc, slots, rows, ctypes.byref(d or desc(K)), None)
    for kw, status in BAD_DESCS:
        assert call(desc(K, **kw)) == status, kw
    assert call(rows=0) == OK and call(rows=0, kn=None) == OK
    for kw in (dict(kn=None), dict(vn=None), dict(kc=None), dict(vc=None), dict(slots=None)):
        assert call(**kw) == NULL, kw
    for kw in (dict(rows=-1), dict(ks=255), dict(vs=-256)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(kn=P + 8), dict(vc=P + 2), dict(ks=260), dict(vs=257)):
        assert call(**kw) == ALIGN, kw


def test_key_bounds_update(K):
    def call(d=None, k=P, b=2 * P, tables=3 * P, lens=4 * P, starts=5 * P, most=7):
        return K.lib().kvc_key_bounds_update(k, b, tables, lens, starts, ctypes.byref(d or desc(K)), most, None)
    for kw, status in BAD_DESCS:
        assert call(desc(K, **kw)) == status, kw
    assert call(most=0) == OK and call(desc(K, num_seqs=0), k=None) == OK
    for kw in (dict(k=None), dict(b=None), dict(tables=None), dict(lens=None)):
        assert call(**kw) == NULL, kw
    assert call(most=-1) == SHAPE and call(starts=None, most=2) == SHAPE
    assert call(k=P + 8) == ALIGN and call(b=P + 2) == ALIGN


def test_block_select(K):
    def call(d=None, q=P, b=2 * P, tables=3 * P, lens=4 * P, starts=5 * P, sel=6 * P, budget=8, first=1, last=1, rows=9, ws=7 * P, ws_bytes=1 << 30):
        return K.lib().kvc_block_select(q, b, tables, lens, starts, sel, budget, first, last, ctypes.byref(d or desc(K)), rows, ws, ws_bytes, None)

    def need(d=None, rows=9, budget=8, first=1, last=1):
        return K.lib().kvc_block_select_workspace_bytes(ctypes.byref(d or desc(K)), rows, budget, first, last)
    for kw, status in BAD_DESCS:
        assert call(desc(K, **kw)) == status and need(desc(K, **kw)) == 0, kw
    for kw in (dict(budget=0), dict(first=-1), dict(last=0), dict(first=4, last=5), dict(first=2 ** 31 - 1, last=2 ** 31 - 1)):
        assert call(**kw) == SHAPE and need(**kw) == 0, kw
    assert call(rows=-1) == SHAPE and call(starts=None) == SHAPE and call(rows=1 << 23) == SHAPE
    assert call(rows=0) == OK and call(desc(K, num_seqs=0)) == OK
    for kw in (dict(q=None), dict(b=None), dict(tables=None), dict(lens=None), dict(sel=None)):
        assert call(**kw) == NULL, kw
    assert call(q=P + 8) == ALIGN and call(b=P + 8) == ALIGN and call(ws=P + 16) == ALIGN
    assert need() > 0 and call(ws=None) == WORKSPACE and call(ws_bytes=need() - 1) == WORKSPACE
    assert need(budget=64) == 0 and need(budget=5, first=4) == 0 and need(desc(K, max_context_len=100)) == 0


def test_paged_attention_selected(K):
    def call(d=None, q=P, k=2 * P, v=3 * P, tables=4 * P, lens=5 * P, starts=6 * P, sel=7 * P, budget=8, scale=0.1, out=8 * P, rows=9, ws=9 * P,
             ws_bytes=1 << 30):
        return K.lib().kvc_paged_attention_selected(q, k, v, tables, lens, starts, sel, budget, scale, out, ctypes.byref(d or desc(K)), rows, ws,
                                                    ws_bytes, None)
    for kw, status in BAD_DESCS:
        assert call(desc(K, **kw)) == status, kw
        assert K.lib().kvc_paged_attention_selected_workspace_bytes(ctypes.byref(desc(K, **kw)), 9, 8) == 0
    for kw in (dict(budget=0), dict(budget=(1 << 26) + 1), dict(rows=-1), dict(rows=1 << 23), dict(starts=None), dict(scale=float("inf")),
               dict(scale=float("nan"))):
        assert call(**kw) == SHAPE, kw
    assert call(rows=0) == OK and call(desc(K, num_seqs=0)) == OK
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(tables=None), dict(lens=None), dict(sel=None), dict(out=None)):
        assert call(**kw) == NULL, kw
    for kw in (dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=P + 8)):
        assert call(**kw) == ALIGN, kw


def test_lists_of_scores_that_do_not_fit(K):
    """Rows of scores are indexed in 32 bits, and many blocks are chosen among by 1024 threads a row."""
    def need(rows, **kw):
        return K.lib().kvc_block_select_workspace_bytes(ctypes.byref(desc(K, **kw)), rows, 8, 1, 1)
    for blocks, fits in ((1 << 30, False), ((1 << 30) - 32, True)):
        d = desc(K, block_size=1, max_blocks_per_seq=blocks)
        assert (need(9, block_size=1, max_blocks_per_seq=blocks) > 0) == fits
        rc = K.lib().kvc_block_select(P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 8, 1, 1, ctypes.byref(d), 9, None, 0, None)
        assert rc == (WORKSPACE if fits else SHAPE)
    hkv = desc(K).num_kv_heads
    for blocks, rows, fits in ((2049, (1 << 22) // hkv, False), (2049, ((1 << 22) - 1) // hkv, True), (2048, (1 << 22) // hkv, True)):
        assert (need(rows, max_blocks_per_seq=blocks) > 0) == fits


def test_a_workspace_does_for_smaller_calls(K):
    """Fewer rows, blocks and kept blocks have more shares and parts each; what was asked for before has room for them."""
    for dtype in (K.KVC_F32, K.KVC_BF16):
        def select(rows, blocks, first=0):
            d = desc(K, dtype=dtype, num_seqs=rows, num_q_heads=8, num_kv_heads=1, max_blocks_per_seq=blocks)
            return K.lib().kvc_block_select_workspace_bytes(ctypes.byref(d), rows, 8, first, 1)
        for rows in (1, 2, 8, 9, 1024, 1025):
            sizes = [select(rows, b) for b in (9, 10, 64, 65, 129, 130, 513, 514, 2048, 2049, 8193, 8194, 65537, 65538, 65539)]
            assert sizes == sorted(sizes) and all(select(rows, b, 3) <= select(rows, b) for b in (65538, 65541, 8194, 8197))
        for blocks in (10, 65538):
            sizes = [select(rows, blocks) for rows in range(1, 1100, 7)]
            assert sizes == sorted(sizes)
        for block_size, hq in ((16, 8), (1, 8), (64, 2), (16, 40)):
            def selected(rows, budget):
                d = desc(K, dtype=dtype, num_seqs=rows, num_q_heads=hq, num_kv_heads=2, block_size=block_size, max_blocks_per_seq=4096)
                return K.lib().kvc_paged_attention_selected_workspace_bytes(ctypes.byref(d), rows, budget)
            for budget in (1, 4, 40, 128, 2000):
                sizes = [selected(rows, budget) for rows in (1, 2, 3, 8, 16, 17, 32, 64, 65, 128, 129, 1000)]
                assert sizes == sorted(sizes)
            for rows in (1, 40, 1000):
                sizes = [selected(rows, budget) for budget in (1, 2, 3, 8, 9, 32, 33, 100, 128, 2000, 4096)]
                assert sizes == sorted(sizes)
