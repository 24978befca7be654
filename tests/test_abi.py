"""The C-ABI library builds, loads without a GPU, and exports every function include/defl.h declares."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def libpath():
    from paper_2609_21102_b200 import build
    return build.build()


def _declared():
    text = open(os.path.join(ROOT, "include", "defl.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(defl_[a-z_0-9]+)\s*\(", text)))


def test_header_declares_the_two_primitives():
    names = _declared()
    assert "defl_polar_batched" in names and "defl_psd_project" in names
    assert len(names) >= 10


def test_library_exports_every_declared_symbol(libpath):
    L = ctypes.CDLL(libpath)
    for name in _declared():
        assert hasattr(L, name), name


def test_binding_lists_the_same_names(libpath):
    from paper_2609_21102_b200 import binding
    assert sorted(binding.EXPORTS) == _declared()
    binding.lib()


def test_status_strings_and_no_device_behaviour(libpath):
    import torch
    L = ctypes.CDLL(libpath)
    L.defl_status_string.restype = ctypes.c_char_p
    for code in (0, -1, -2, -3, -4):
        assert len(L.defl_status_string(code)) > 0
    assert L.defl_polar_workspace_bytes(0, 4, 4, 0, 0, 0) == 0
    L.defl_polar_workspace_bytes.restype = ctypes.c_size_t
    assert L.defl_polar_workspace_bytes(2, 128, 256, 0, 4, 4) > 2 * 128 * 256 * 2
    if not torch.cuda.is_available():
        h = ctypes.c_void_p()
        # no CPU fallback: without a device the context cannot even be created
        assert L.defl_create(ctypes.byref(h), 0) == -3
        assert not h.value


def test_shape_groups_and_stacking():
    """Host-side grouping of a parameter list by stored shape (no GPU, no arithmetic)."""
    import torch
    from paper_2609_21102_b200 import grouping
    shapes = [(8, 4), (4, 8), (8, 4), (3,), (8, 4), (4, 8), (2, 2, 2)]
    g = grouping.shape_groups(shapes)
    assert list(g.items()) == [((8, 4), [0, 2, 4]), ((4, 8), [1, 5])]
    ts = [torch.full(s, float(i)) for i, s in enumerate(shapes)]
    buf, views = grouping.stack_group(ts, g[(8, 4)])
    assert buf.shape == (3, 8, 4) and [float(v[0, 0]) for v in views] == [0.0, 2.0, 4.0]
    views[1].add_(1.0)                      # a view writes through to the stacked buffer
    assert float(buf[1, 3, 3]) == 3.0
    with pytest.raises(ValueError):
        grouping.stack_group(ts, [0, 1])


def test_deflation_cutoff_switch():
    """Section 4, "Deflation cutoff": deflation during the first fraction of the optimizer steps, the plain step after;
    the step helper passes k = 0 past the cutoff (a recording stand-in for the context, no GPU)."""
    from paper_2609_21102_b200 import grouping
    assert [grouping.deflation_active(t, 10, 0.3) for t in range(10)] == [True] * 3 + [False] * 7
    assert all(grouping.deflation_active(t, 10, 1.0) for t in range(10))
    assert not any(grouping.deflation_active(t, 10, 0.0) for t in range(10))
    assert [grouping.deflation_active(t, 5, 0.5) for t in range(5)] == [True, True, True, False, False]   # 2.5 steps
    with pytest.raises(ValueError):
        grouping.deflation_active(0, 10, 1.5)

    class Recorder:
        def __init__(self):
            self.calls = []

        def defl_muon_step_batched(self, W, M, G, lr, mu, k, p, J, sched, **kw):
            self.calls.append((k, p, J))
    rec = Recorder()
    weights = {(1600, 6400): "W"}
    for t in range(4):
        grouping.muon_step_groups(rec, weights, {(1600, 6400): "M"}, {}, 0.02, 0.95, 0.02, 0.01, 2, [[1.0, 0.0, 0.0]],
                                  step=t, total_steps=4, cutoff=0.5)
    assert rec.calls == [(32, 16, 2), (32, 16, 2), (0, 16, 2), (0, 16, 2)]


def test_window_ratios_follow_the_algorithms(libpath):
    """Algorithm 3 line 1 (r = ceil(w m), r' = min{m, r + ceil(delta m)}) and Algorithm 2's inputs (r = ceil(w n),
    K = ceil(w' n)), worked by hand."""
    import pytest
    from paper_2609_21102_b200 import binding
    assert binding.defl_polar_window(1600, 6400, 0.02, 0.01) == (32, 16)
    assert binding.defl_polar_window(6400, 1600, 0.02, 0.01) == (32, 16)          # the short side counts
    assert binding.defl_polar_window(768, 3072, 0.01, 0.0105) == (8, 9)           # ceil(7.68) = 8, ceil(8.064) = 9
    assert binding.defl_polar_window(40, 40, 0.5, 0.9) == (20, 20)                # r' capped at the short side
    assert binding.defl_polar_window(40, 64, 1.0, 0.0) == (39, 0)                 # r capped at m - 1
    assert binding.defl_psd_window(4096, 8 / 4096, 16 / 4096) == (8, 16)
    assert binding.defl_psd_window(640, 0.025, 0.05) == (16, 32)
    with pytest.raises(binding.DeflError) as e:
        binding.defl_psd_window(5000, 0.025, 0.05)                                 # K = 250 exceeds the widest basis
    assert e.value.code == -2
    with pytest.raises(binding.DeflError) as e:
        binding.defl_polar_window(128, 256, -0.1, 0.0)
    assert e.value.code == -1


def test_pointers_that_are_not_multiples_of_their_elements_are_refused(libpath):
    """Decided on the host before anything is launched, so that a block of zeros may stand in for the context."""
    import numpy as np
    from paper_2609_21102_b200 import binding
    L = binding.lib()
    room = ctypes.create_string_buffer(1 << 20)
    at = 1 << 12                                             # (an address that nothing reads)
    fine = dict(p=at, g=at, m=at, v=at, m_scale=at, v_scale=at, copy=at, n=10, p_dtype=binding.F32, g_dtype=binding.F32, state_bits=8)

    class Opts(ctypes.Structure):
        _fields_ = [(x, ctypes.c_double) for x in ("lr", "beta1", "beta2", "eps", "weight_decay")] + \
                   [("step", ctypes.c_int64)] + [(x, ctypes.c_void_p) for x in ("step_dev", "lr_dev", "grad_scale")] + \
                   [("seed", ctypes.c_uint64), ("stochastic", ctypes.c_int)]

    def adamw(opts=None, **kw):
        t = np.zeros(1, dtype=binding._ADAMW_TENSOR)
        for key, value in {**fine, **kw}.items():
            t[key] = value
        o = Opts(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, **(opts or {}))
        return L.defl_adamw_step(room, ctypes.c_void_p(t.ctypes.data), 1, ctypes.byref(o))
    for kw in (dict(p=at + 2), dict(g=at + 2), dict(p=at + 1, p_dtype=binding.BF16), dict(g=at + 1, g_dtype=binding.BF16), dict(copy=at + 1),
               dict(m_scale=at + 2), dict(v_scale=at + 1), dict(m=at + 2, state_bits=32), dict(v=at + 1, state_bits=32),
               dict(opts=dict(step_dev=at + 4)), dict(opts=dict(lr_dev=at + 2)), dict(opts=dict(grad_scale=at + 2))):
        assert adamw(**kw) == -1, kw

    class Norm(ctypes.Structure):
        _fields_ = [("x", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int)]

    def norm(x=at, dtype=binding.F32, out=at, step=at, work=at):
        t = Norm(x, 10, dtype)
        return L.defl_grad_norm(room, ctypes.byref(t), 1, ctypes.c_float(1.0), ctypes.c_void_p(out), ctypes.c_void_p(step), ctypes.c_void_p(work))
    for kw in (dict(x=at + 2), dict(x=at + 1, dtype=binding.BF16), dict(out=at + 2), dict(step=at + 4), dict(work=at + 4)):
        assert norm(**kw) == -1, kw
    # nvfp4's matrix scale, in each of the three calls
    q, bad = (ctypes.c_void_p * 3)(at, at, at), (ctypes.c_void_p * 3)(at, at, at + 2)
    i64, p = ctypes.c_int64, ctypes.c_void_p
    for rows, cols in ((bad, None), (None, bad), (q, bad)):
        assert L.defl_mx4_quantize(room, p(at), binding.F32, 1, 4, 4, i64(4), i64(16), 1, rows, cols, p(at)) == -1
    assert L.defl_mx4_dequantize(room, bad, 1, 4, 4, 1, p(at), binding.F32) == -1
    for a, b in ((bad, q), (q, bad)):
        assert L.defl_mx4_gemm(room, a, b, 1, 4, 4, 4, 0, 1, ctypes.c_float(1.0), p(at), i64(4), i64(16), binding.F32, None) == -1
    # the Muon step's factor
    schedule = (ctypes.c_float * 3)(1.0, 0.0, 0.0)
    f = ctypes.c_float
    assert L.defl_muon_step_scaled(room, p(at), binding.F32, p(at), p(at), 1, 4, 4, binding.F32, f(0.1), f(0.9), 0, f(0.0), f(1.0), 1, 1, 1,
                                   schedule, 1, None, None, p(at + 2)) == -1


def test_native_module_follows_its_torch_and_can_be_missing(libpath, monkeypatch, tmp_path):
    """Built again when the torch or the Python it was built with is another; where no compiler or header is found, the library's build stands
    and an old module does not. (The commands are recorded, not run.)"""
    import shutil
    import torch
    from paper_2609_21102_b200 import build
    assert build.build_native() == build.NATIVE and os.path.exists(build.NATIVE)
    target, ran = str(tmp_path / "_native.so"), []

    def run(cmd, check):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(build, "NATIVE", target)
    monkeypatch.setattr(build.subprocess, "run", run)
    assert build.build_native() == target and len(ran) == 1
    assert build.build_native() == target and len(ran) == 1
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build.build_native() == target and len(ran) == 2
    assert build.build_native() == target and len(ran) == 2
    monkeypatch.setattr(shutil, "which", lambda name: None)
    assert build.build_native() == target                    # nothing to do
    monkeypatch.setattr(torch, "__version__", "0.0.2")
    with pytest.warns(UserWarning, match=r"no g\+\+"):
        assert build.build_native() is None
    assert len(ran) == 2 and not os.path.exists(target)


def test_options_do_not_grow(tmp_path):
    """defl_opts has no size field: a caller built against an earlier header passes one that ends with poly_terms, and no call may read on."""
    import subprocess
    from paper_2609_21102_b200 import binding
    src, exe = tmp_path / "size.c", tmp_path / "size"
    src.write_text('#include <stddef.h>\n#include <stdint.h>\n#include <stdio.h>\n#include "defl.h"\n'
                   'int main(void) { printf("%zu %zu %zu\\n", sizeof(defl_opts), offsetof(defl_opts, poly_terms), _Alignof(defl_opts)); return 0; }\n')
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    size, last, align = (int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    assert size == -(-(last + 4) // align) * align == ctypes.sizeof(binding.DeflOpts)
