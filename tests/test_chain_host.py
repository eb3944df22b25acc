"""The composition of the recurrence's segment maps on the CPU
(tests/sanitize/chain_driver.cpp, with AddressSanitizer and
UndefinedBehaviorSanitizer on the host code): a run's map has the same bits
whichever fans' maps are there in time."""

import os
import subprocess

import pytest

from test_host_sanitizers import CLANG, HIPCC, ROOT, _run

pytestmark = pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="needs hipcc")


def test_composition_of_segment_maps(tmp_path):
    src, obj, exe = os.path.join(ROOT, "tests", "sanitize", "chain_driver.cpp"), str(tmp_path / "d.o"), str(tmp_path / "d")
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature",
                    "-Xclang", "-packed-fp32-ops", "-Xarch_host", "-fno-omit-frame-pointer",
                    "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-c", src, "-o", obj],
                   check=True, capture_output=True, text=True)
    subprocess.run([CLANG, "-fsanitize=address,undefined", obj, "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True, capture_output=True, text=True)
    _run(exe, env_extra={"ASAN_OPTIONS": "detect_leaks=0:abort_on_error=0",
                         "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1"})
