"""The host side of the sequence-core entry points (argument checks, size
queries, no-op paths), built with AddressSanitizer + UndefinedBehaviorSanitizer
and driven on the CPU by tests/sanitize/seq_driver.cpp; and the binding's own
checks that need no GPU.  The launchers that compute the sizes are host code of
the kernel files, so these are built with the sanitizers too (host side only:
each -fsanitize= on a hipcc line follows -Xarch_host)."""

import glob
import os
import subprocess

import pytest
import torch

from paper_2205_01435_amd import _lib as wm
from test_host_sanitizers import BUILD, CLANG, HIPCC, PKG, ROOT, _run

pytestmark = pytest.mark.skipif(
    not (os.path.exists(HIPCC) and os.path.exists(CLANG) and glob.glob(os.path.join(BUILD, "wm_linrec.o"))),
    reason="needs hipcc and the library's object files (run __graft_entry__.build())")


def test_argument_checks_under_sanitizers(tmp_path):
    mine = ["wm_api.cpp", "wm_profile.cpp", "wm_clip.hip"]
    flags = ["-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-Xarch_host", "-fno-omit-frame-pointer",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    objs = []
    for src in [os.path.join(PKG, "csrc", f) for f in mine] + [os.path.join(ROOT, "tests", "sanitize", "seq_driver.cpp")]:
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
    x = torch.zeros(2, 3, 4)
    with pytest.raises(ValueError):
        wm.embed(x[0], torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        wm.layer_norm(x)
    with pytest.raises(ValueError):
        wm.linrec(x, x)
    with pytest.raises(ValueError):
        wm.ClipPlan([x])
    with pytest.raises(ValueError):
        wm.ClipPlan([])
