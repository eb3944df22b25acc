"""The host side of the attending-core entry points (argument checks, size
queries, no-op paths, the rotation's table), built with AddressSanitizer +
UndefinedBehaviorSanitizer and driven on the CPU by
tests/sanitize/attend_driver.cpp; and the binding's own checks that need no GPU.
(Host side only: each -fsanitize= on a hipcc line follows -Xarch_host.)"""

import glob
import os
import subprocess

import pytest
import torch

from paper_2205_01435_amd import _lib as wm
from test_host_sanitizers import BUILD, CLANG, HIPCC, PKG, ROOT, _run

pytestmark = pytest.mark.skipif(
    not (os.path.exists(HIPCC) and os.path.exists(CLANG) and glob.glob(os.path.join(BUILD, "wm_linattn.o"))),
    reason="needs hipcc and the library's object files (run __graft_entry__.build())")


def test_argument_checks_under_sanitizers(tmp_path):
    mine = ["wm_api.cpp", "wm_profile.cpp", "wm_qknorm.hip"]
    flags = ["-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-Xarch_host", "-fno-omit-frame-pointer",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    objs = []
    for src in [os.path.join(PKG, "csrc", f) for f in mine] + [os.path.join(ROOT, "tests", "sanitize", "attend_driver.cpp")]:
        o = str(tmp_path / (os.path.splitext(os.path.basename(src))[0] + ".o"))
        subprocess.run([HIPCC, *flags, "-c", src, "-o", o], check=True, capture_output=True, text=True)
        objs.append(o)
    skip = {os.path.splitext(f)[0] + ".o" for f in mine}
    kernels = [o for o in sorted(glob.glob(os.path.join(BUILD, "*.o"))) if os.path.basename(o) not in skip]
    exe = str(tmp_path / "driver")
    subprocess.run([CLANG, "-fsanitize=address,undefined", *objs, *kernels, "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True, capture_output=True, text=True)
    _run(exe, env_extra={"ASAN_OPTIONS": "detect_leaks=0:abort_on_error=0",
                         "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1"})


def test_host_tensors_are_refused():
    x = torch.zeros(2, 3, 4, 5)
    pos = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        wm.qk_norm(x[0], x[0], pos, None)
    with pytest.raises(ValueError):
        wm.qk_norm_grad(x[0], x[0], x[0], x[0], pos, None)
    with pytest.raises(ValueError):
        wm.linattn(x, x, x, torch.zeros(4))
    with pytest.raises(ValueError):
        wm.linattn_grad(x, x, x, torch.zeros(4), x)
    with pytest.raises(ValueError):
        wm.glu(x[0, 0], torch.zeros(6, 5))
    with pytest.raises(ValueError):
        wm.glu_grad(x[0, 0], torch.zeros(6, 5), torch.zeros(4, 3))


def test_the_table_needs_no_gpu():
    t = wm.Rotary(8, 10000.0, device="cpu").table
    assert t.dtype == torch.int64 and t.shape == (4,)
    assert abs(int(t[0]) / 2.0 ** 64 - 0.15915494309189535) < 1e-15
    assert wm.Rotary(0, device="cpu").R == 0
    for R, base in ((7, 10.0), (258, 10.0), (8, 0.5)):
        with pytest.raises(wm.WmError):
            wm.Rotary(R, base, device="cpu")
