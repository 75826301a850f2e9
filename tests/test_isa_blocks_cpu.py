"""What the compiler made of the publication protocols of block choice and attention over chosen blocks (no GPU needed): the count that tells
the last workgroup of a row that all parts are there comes behind a wait for this workgroup's own stores and a barrier; and the kernels that
load tiles straight into LDS do not read a tile before they have waited for it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2503_13773_amd import build as B


def _kernels(tmp_path, source, name):
    hipcc = B._hipcc()
    if not (shutil.which(hipcc) or os.path.exists(hipcc)):
        pytest.skip("hipcc not available")
    out = tmp_path / "kernels.s"
    r = subprocess.run([hipcc, *[f for f in B.FLAGS if f != "-fPIC"], "--cuda-device-only", "-S", os.path.join(B.CSRC, source), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    kernels, at = {}, None
    for ln in out.read_text().splitlines():
        m = re.match(rf"^(_ZN\S*{name}\S*):", ln)
        if m:
            at = kernels.setdefault(m.group(1), [])
        elif ln.startswith(".Lfunc_end"):
            at = None
        elif at is not None:
            at.append(ln.strip())
    return kernels


@pytest.mark.parametrize("source,name,store,least", [("block_select.hip", "block_scores_kernel", r"global_store_dword\b.* sc1", 4),
                                                     ("paged_attention_selected.hip", "pa_selected_mfma_kernel", r"buffer_store_dword.* sc1", 12),
                                                     ("paged_attention_selected.hip", "pa_selected_valu_kernel", r"global_store_dword\b.* sc1", 24)])
def test_parts_are_published_before_they_are_counted(tmp_path, source, name, store, least):
    checked = 0
    for kernel, body in _kernels(tmp_path, source, name).items():
        for i in [i for i, ln in enumerate(body) if ln.startswith("global_atomic_add")]:
            before = [j for j in range(i) if re.match(store, body[j])]
            assert before, (kernel, body[i])
            between = body[before[-1] + 1:i]
            waits = [j for j, ln in enumerate(between) if re.match(r"s_waitcnt\b.*vmcnt\(0\)", ln)]
            assert waits, f"{kernel}: no wait for the part's stores before `{body[i]}`"
            assert any(ln.startswith("s_barrier") for ln in between[waits[0]:]), f"{kernel}: no barrier between the wait and `{body[i]}`"
            checked += 1
    assert checked >= least, checked


def test_tiles_are_waited_for_before_they_are_read(tmp_path):
    """In the order of the code: between the loads of a tile into LDS and the next reads from LDS of their kind stands a wait that leaves at most one
    tile's loads of the other kind under way, and the compiler has added no wait for all loads inside the loop (Q's would be one)."""
    for name in ("pa_selected_wave_kernel", "pa_selected_mfma_kernel"):
        kernels = _kernels(tmp_path, "paged_attention_selected.hip", name)
        assert kernels
        for kernel, body in kernels.items():
            loads = 4 if "ILi64E" in kernel else 8
            first = next(i for i, ln in enumerate(body) if ln.startswith("global_load_lds_dwordx4"))
            last = max(i for i, ln in enumerate(body) if ln.startswith("global_load_lds_dwordx4"))
            k_reads = [i for i in range(first, last) if body[i].startswith("ds_read_b128")]
            v_reads = [i for i, ln in enumerate(body) if i > first and ln.startswith("ds_read_b64_tr_b16")]
            assert k_reads and v_reads, kernel
            for at in (k_reads[0], v_reads[0]):
                waits = [ln for ln in body[first:at] if ln.startswith("s_waitcnt") and "vmcnt" in ln]
                assert waits and any(f"vmcnt({loads})" in w or "vmcnt(0)" in w for w in waits), (kernel, body[at], waits[-3:])
            # loop: from the first K read to the last load; the waits of the loop are ours
            inside = [ln for ln in body[k_reads[0]:last] if ln.startswith("s_waitcnt") and "vmcnt" in ln]
            ours = {f"vmcnt({loads})", "vmcnt(0)"}
            assert all(any(o in w for o in ours) for w in inside) and sum("vmcnt(0)" in w for w in inside) <= 1, (kernel, inside)


def test_bounds_are_waited_for_before_they_are_read(tmp_path):
    """The loop that takes bounds from a stage in LDS waits for all loads first, and has read all before the next set is asked for."""
    staged = 0
    for kernel, body in _kernels(tmp_path, "block_select.hip", "block_scores_kernel").items():
        loads = [i for i, ln in enumerate(body) if ln.startswith("global_load_lds_dwordx4")]
        if not loads:
            continue
        staged += 1
        reads = [i for i in range(loads[0], loads[-1]) if body[i].startswith("ds_read_b128")]
        assert reads, kernel
        before = [ln for ln in body[loads[0]:reads[0]] if ln.startswith("s_waitcnt") and "vmcnt(0)" in ln]
        again = next(i for i in loads if i > reads[0])
        done = [i for i in range(reads[0], again) if body[i].startswith("s_waitcnt") and "lgkmcnt(0)" in body[i]]
        assert before and done and max(r for r in reads if r < again) < max(done), kernel
        assert not [r for r in reads if again < r < loads[-1]], kernel
    assert staged >= 8
