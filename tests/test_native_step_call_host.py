"""The native calls of norms, rotary positions and the vocabulary loss on the CPU: csrc/call.cpp built for host tensors, with its allocations and the wrapping of
its results watched, against entries that only count their calls."""
import ctypes
import gc
import importlib.util
import os
import subprocess
import sys
import weakref

import numpy as np
import pytest
import torch

from paper_2502_08141_amd import build

_WATCH = """
extern "C" { int watch_empties, watch_held, watch_fail, watch_after; void (*watch_hook)(); }
static at::Tensor watched_empty(at::IntArrayRef sizes, const at::TensorOptions& o) {
    ++watch_empties; watch_held += PyGILState_Check();
    if (watch_hook) watch_hook();
    return at::empty(sizes, o);
}
static PyObject* watched_wrap(at::Tensor t) {
    if (watch_fail && watch_after-- <= 0) {
        if (watch_fail == 1) throw std::bad_alloc();
        PyErr_NoMemory();
        return nullptr;
    }
    return THPVariable_Wrap(std::move(t));
}
"""
M, N, V, HEADS, KV, D, ROT = 5, 64, 100, 4, 2, 32, 24
HOOK = ctypes.CFUNCTYPE(None)


@pytest.fixture(scope="module")
def native(tmp_path_factory):
    d = tmp_path_factory.mktemp("call")
    text = open(os.path.join(build.CSRC, "call.cpp")).read()
    for old, new, least in (("t.is_cuda()", "t.is_cpu()", 1), ("!x.is_cuda()", "!x.is_cpu()", 1), ("(void*)c10::hip::getCurrentHIPStream().stream()", "nullptr", 1),
                            ("t.get_device() == c10::hip::current_device()", "true", 1), ("at::empty(", "watched_empty(", 1), ("THPVariable_Wrap(", "watched_wrap(", 5)):
        assert text.count(old) >= least, old
        text = text.replace(old, new)
    text = text.replace("namespace {\n", _WATCH + "namespace {\n", 1)
    (d / "call.cpp").write_text(text)
    so = str(d / "_lowra_call.so")
    subprocess.run([a if a != "-O2" else "-O0" for a in build.call_command(str(d / "call.cpp"), so)], check=True)
    spec = importlib.util.spec_from_file_location("_lowra_call", so)
    call = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(call)

    vp, i, f, n = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib = type("lib", (), {"calls": 0, "status": 0, "keep": [], "seen": None})

    def entry(*types):
        def count(*args):
            lib.calls += 1
            lib.seen = lib.look(args) if lib.look else args
            return lib.status
        lib.keep.append(ctypes.CFUNCTYPE(i, *types)(count))
        return ctypes.cast(lib.keep[-1], vp).value

    lib.look = None
    call.init_step(entry(i, i, i, vp, vp, vp, f, vp, vp), entry(i, i, i, vp, vp, vp, f, vp, vp, vp, vp, vp, n, vp), entry(i, vp, i, i, i, i, vp, vp, f, i, vp),
                   entry(i, i, i, vp, vp, vp, vp, vp, vp, vp, vp, n, vp))
    handle = ctypes.CDLL(so)
    watch = {k: ctypes.c_int.in_dll(handle, "watch_" + k) for k in ("empties", "held", "fail", "after")}
    watch["hook"] = vp.in_dll(handle, "watch_hook")
    return call, lib, watch


def _reset(lib, watch):
    lib.calls, lib.status, lib.look = 0, 0, None
    for v in watch.values():
        v.value = 0


def _calls(call):
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    x, w, ws, h, W = z(M, N), z(N), z(512, dtype=torch.uint8), z(M, N), z(V, N)
    targets, weights = z(M, dtype=torch.int32), z(M, dtype=torch.float32)
    q, k, positions, turns = z(M, HEADS, D), z(M, KV, D), z(M, dtype=torch.int32), z(ROT // 2, dtype=torch.int64)
    back = lambda *want: (lambda: call.norm_bwd(x, x, w, 1, 1e-5, None, *want, ws))
    return {"norm_fwd": (lambda: call.norm_fwd(x, w, None, 0, 1e-5), [(M, N)]),
            "norm_bwd": (back(True, True, True), [(M, N), (N,), (N,)]),
            "norm_bwd without dX": (back(False, True, True), [None, (N,), (N,)]),
            "norm_bwd of dbias": (back(False, False, True), [None, None, (N,)]),
            "norm_bwd of dX": (back(True, False, False), [(M, N), None, None]),
            "rope": (lambda: call.rope(q, positions, turns, 0, False, 1.0), [(M, HEADS, D)]),
            "rope of a list": (lambda: call.rope([q, k], positions, turns, 0, True, 1.0), [(M, HEADS, D), (M, KV, D)]),
            "rope of a tuple": (lambda: call.rope((q, k, q, k), positions, turns, 1, True, 1.0), [(M, HEADS, D), (M, KV, D)] * 2),
            "vocab_loss": (lambda: call.vocab_loss(h, W, targets, weights, True, ws), [(M,), (M,), (M, N)]),
            "vocab_loss alone": (lambda: call.vocab_loss(h, W, targets, None, False, ws), [(M,), (M,), None])}


NAMES = ["norm_fwd", "norm_bwd", "norm_bwd without dX", "norm_bwd of dbias", "norm_bwd of dX", "rope", "rope of a list", "rope of a tuple", "vocab_loss", "vocab_loss alone"]


def _tensors():
    gc.collect()
    return sum(type(o) is torch.Tensor for o in gc.get_objects())


@pytest.mark.parametrize("which", NAMES)
def test_allocations_and_failures(native, which):
    call, lib, watch = native
    run, shapes = _calls(call)[which]
    _reset(lib, watch)
    res = run()
    assert [None if t is None else tuple(t.shape) for t in (res if isinstance(res, (tuple, list)) else (res,))] == shapes and lib.calls == 1
    del res
    # other threads run while an output is allocated
    wanted = sum(s is not None for s in shapes)
    assert watch["empties"].value == wanted and watch["held"].value == 0
    # "nothing launched" is what None says, whichever output cannot be wrapped, and nothing stays behind
    before, nones = _tensors(), sys.getrefcount(None)
    for after in range(wanted):
        for watch["fail"].value in (1, 2):
            watch["after"].value = after
            assert run() is None and lib.calls == 1
    assert _tensors() == before and abs(sys.getrefcount(None) - nones) < 4
    watch["fail"].value = 0
    lib.status = 4
    for i in range(3):
        assert run() == 4 and lib.calls == 2 + i
    assert _tensors() == before


def test_what_is_left_to_python(native):
    """Nothing is launched for what lowra.py has to look at itself."""
    call, lib, watch = native
    _reset(lib, watch)
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    x, w, ws, h, W, t, f = z(M, N), z(N), z(512, dtype=torch.uint8), z(M, N), z(V, N), z(M + 1, dtype=torch.int32), z(M + 1, dtype=torch.float32)
    p, turns, q = z(M, dtype=torch.int32), z(ROT // 2, dtype=torch.int64), z(M, HEADS, D)
    for bad in ((x.float(), w, None, 0, 1e-5), (x, z(N + 8), None, 0, 1e-5), (x[:, :8], None, None, 0, 1e-5), (x, w, None, 0, 1), (x, w, None, 0.0, 1e-5), (None, w, None, 0, 1e-5)):
        assert call.norm_fwd(*bad) is None
    for bad in ((x, None, w, 0, 1e-5, None, True, True, True, ws), (x, x, w, 0, 1e-5, z(M, 8), True, True, True, ws), (x, x, w, 0, 1e-5, None, 1, True, True, ws),
                (x, x, w, 0, 1e-5, None, True, True, True, None)):
        assert call.norm_bwd(*bad) is None
    for bad in ((q[0], p, turns, 0, False, 1.0), ([], p, turns, 0, False, 1.0), ([q] * 5, p, turns, 0, False, 1.0), ([q, None], p, turns, 0, False, 1.0), (q, p[1:], turns, 0, False, 1.0),
                ([q, z(M, 2, D + 2)], p, turns, 0, False, 1.0), (q.transpose(1, 2), p, turns, 0, False, 1.0), (q, p, turns, 0, 0, 1.0)):
        assert call.rope(*bad) is None
    for bad in ((h, W, t, None, True, ws), (h, W[:, :8], t[:M], None, True, ws), (h, W, t[:M].long(), None, True, ws), (h, W, t[:M], f, True, ws), (h, W, t[:M], None, 1, ws),
                (h, W, t[1:], None, True, ws), (h, W, t[:M], f[1:], True, ws)):
        assert call.vocab_loss(*bad) is None
    assert lib.calls == 0


def test_list_that_another_thread_empties(native):
    """The interpreter's lock is given up while outputs are allocated: a list that loses its tensors meanwhile does not free what the library is about to read."""
    call, lib, watch = native
    _reset(lib, watch)
    data = np.zeros((M, HEADS, D), np.int16)
    gone = weakref.ref(data)
    xs = [torch.from_numpy(data).view(torch.bfloat16), torch.zeros(M, KV, D, dtype=torch.bfloat16)]
    del data
    hook = HOOK(lambda: xs.clear())
    watch["hook"].value = ctypes.cast(hook, ctypes.c_void_p).value
    lib.look = lambda args: gone() is not None
    res = call.rope(xs, torch.zeros(M, dtype=torch.int32), torch.zeros(ROT // 2, dtype=torch.int64), 0, False, 1.0)
    watch["hook"].value, lib.look = 0, None
    assert len(res) == 2 and lib.calls == 1 and not xs
    assert lib.seen is True
    del res
    gc.collect()
    assert gone() is None
