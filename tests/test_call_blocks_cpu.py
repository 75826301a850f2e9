"""The native calls of the operators around the cache's blocks on CPU tensors: kvc_call.cpp compiled with CPU tensors taken for
device tensors and bound to functions that only record that they were called."""
import os
import subprocess
import sys
import textwrap

import pytest

import paper_2503_13773_amd.build as B

SETUP = """
import ctypes, importlib.machinery, importlib.util, sys, warnings
import torch
warnings.simplefilter("ignore")
loader = importlib.machinery.ExtensionFileLoader("kvc_call", sys.argv[1])
C = importlib.util.module_from_spec(importlib.util.spec_from_loader("kvc_call", loader))
loader.exec_module(C)
vp, sz, f, i32, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_int32, ctypes.c_int64
called, args_of, need = [], {}, {"bytes": 0}
def stub(name, result, *types):
    def record(*args):
        called.append(name)
        args_of[name] = args
        return need["bytes"] if name == "bytes" else 0
    return ctypes.CFUNCTYPE(result, *types)(record)
stubs = [stub("extend", i32, *[vp] * 5, i32, vp, vp, vp), stub("write", i32, vp, vp, i64, i64, vp, vp, vp, i32, vp, vp),
         stub("bounds", i32, *[vp] * 6, i32, vp), stub("bytes", sz, vp, *[i32] * 4),
         stub("select", i32, *[vp] * 6, i32, i32, i32, vp, i32, vp, sz, vp), stub("bytes", sz, vp, i32, i32),
         stub("selected", i32, *[vp] * 7, i32, f, vp, vp, i32, vp, sz, vp)]
C.bind_blocks(*(ctypes.cast(s, vp).value for s in stubs))
bf, i4 = torch.bfloat16, torch.int32
def ints(*shape):
    return torch.zeros(*shape, dtype=i4)
q, k, bounds = torch.zeros(7, 8, 64, dtype=bf), torch.zeros(5, 2, 16, 64, dtype=bf), torch.zeros(5, 2, 2, 64, dtype=bf)
qkv = torch.zeros(7, 12, 64, dtype=bf)
bt, cl, qs, slots, sel = ints(3, 4), ints(3), ints(4), torch.zeros(7, dtype=torch.int64), ints(7, 2, 6)
update = (ints(4), ints(3), ints(3), ints(1), torch.zeros(9, dtype=torch.int64), ints(9), ints(9))
ws = torch.zeros(4096, dtype=torch.uint8)
good = {"extend": [bt, cl, ints(3), ints(3), ints(11), 16, update, -1, 0],
        "write": [qkv[:, 8:10], qkv[:, 10:], k, k, slots, -1, 0],
        "bounds": [k, bounds, bt, cl, qs, 5, -1, 0],
        "select": [q, bounds, bt, cl, qs, 6, 16, 1, 2, 0, sel, ws, -1, 0],
        "selected": [q, k, k, bt, cl, qs, sel, 0.1, q.clone(), 0, ws, -1, 0]}
def call(name, **change):
    args = list(good[name])
    for at, value in change.items():
        args[int(at[1:])] = value
    called.clear()
    rc = getattr(C, name)(*args)
    ran = [c for c in called if c != "bytes"]
    assert rc == (0 if ran else None), (name, rc, called)   # None: the library has not been called
    return bool(ran)
for name in good:
    assert call(name), name
"""


@pytest.fixture(scope="module")
def module(tmp_path_factory):
    folder = tmp_path_factory.mktemp("kvc_call")
    source = folder / "kvc_call_cpu.cpp"
    source.write_text(open(os.path.join(B.CSRC, "kvc_call.cpp")).read().replace("is_cuda()", "is_cpu()"))
    return B.build_call_module(source=str(source), out=str(folder / "kvc_call.so"))


def run(module, body):
    r = subprocess.run([sys.executable, "-c", SETUP + textwrap.dedent(body), module], cwd=B.ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])


def test_any_other_tensor_is_left_to_the_general_path(module):
    """Each tensor in turn: of another type, size, device, dimension, strided, a view of nothing, no tensor at all."""
    run(module, """
        class Sub(torch.Tensor):
            pass
        for name, args in good.items():
            for i, a in enumerate(args):
                if not isinstance(a, torch.Tensor):
                    continue
                bad = [a.double(), a.unsqueeze(0), a.as_subclass(Sub), torch.empty_like(a, device="meta"), None, 3, "x"]
                if a is not ws:
                    bad += [torch.cat([a, a[:1]]), torch.zeros(*a.shape[:-1], 2 * a.shape[-1], dtype=a.dtype)[..., ::2], torch.nested.nested_tensor([a])]
                else:
                    bad = [torch.empty_like(a, device="meta"), a[::2], 3]
                if (name, i) in (("extend", 4), ("select", 1)):   # a longer free list is one, and a larger pool
                    bad = [x for x in bad if not (isinstance(x, torch.Tensor) and not x.is_nested and x.shape == (len(a) + 1, *a.shape[1:]))]
                for x in bad:
                    if x is None and (name, i) in (("extend", 3), ("bounds", 4), ("select", 4), ("selected", 5)):
                        continue
                    assert not call(name, **{f"a{i}": x}), (name, i, x)
        for i, a in enumerate(update):
            for x in (a.double(), a[None], torch.cat([a, a]), torch.empty_like(a, device="meta"), None, 5):
                if i != 4 or not isinstance(x, torch.Tensor) or x.shape != (18,):
                    assert not call("extend", a6=update[:i] + (x,) + update[i + 1:]), (i, x)
        for x in (update[:6], list(update), None, update + (ints(1),)):
            assert not call("extend", a6=x)
    """)


def test_numbers_devices_and_what_may_be_none(module):
    run(module, """
        for name, ints_at in (("extend", (5,)), ("bounds", (5,)), ("select", (5, 6, 7, 8, 9)), ("selected", (9,))):
            for i in ints_at:
                for x in (2 ** 31, -2 ** 31 - 1, 2 ** 70, 1.0, "1", None, torch.tensor(1)):
                    assert not call(name, **{f"a{i}": x}), (name, i, x)
        for x in (10 ** 400, "0.1", None, 1j):
            assert not call("selected", a7=x)
        assert call("selected", a7=1)
        for name, args in good.items():
            at = len(args) - 2
            assert not call(name, **{f"a{at}": 0}) and not call(name, **{f"a{at}": None})   # tensors of another device
            C_args = args[:-1]
            assert getattr(C, name)(*C_args) is None and getattr(C, name)(*args, 0) is None and getattr(C, name)() is None
        assert call("extend", a3=None) and args_of["extend"][3] is None
        assert call("bounds", a4=None) and call("select", a4=None) and call("selected", a5=None)
        assert call("select", a11=None) and call("selected", a10=None)    # none is needed
        need["bytes"] = 64
        assert not call("select", a11=None) and not call("selected", a10=None)   # one is: the general path allocates it
        assert call("select") and call("selected")
    """)


def test_rows_that_lie_apart(module):
    run(module, """
        assert call("write") and args_of["write"][2:4] == (12 * 64, 12 * 64)
        new = torch.zeros(7, 2, 64, dtype=bf)
        assert call("write", a0=new, a1=new) and args_of["write"][2:4] == (128, 128)
        assert call("write", a0=new[:1], a1=new[:1], a4=slots[:1]) and args_of["write"][2:4] == (0, 0)
        for x in (new[:1].expand(7, 2, 64), torch.zeros(7, 64, 2, dtype=bf).transpose(1, 2), torch.zeros(2, 7, 64, dtype=bf).transpose(0, 1),
                  torch.zeros(7 * 64 + 64, dtype=bf).as_strided((7, 2, 64), (64, 64, 1))):
            assert not call("write", a0=x) and not call("write", a1=x)
    """)
