"""The kernels and the C ABI of fla_seq.h, built for the CPU and run against the fp64 forms.

As in ``test_kernel_host_emu``: the unmodified sources are compiled as host C++ against a stand-in for the HIP
runtime (the work items of a block are coroutines that change over at barriers; lane permutations exchange their
operands around a barrier over the wave), with AddressSanitizer and UndefinedBehaviorSanitizer, and run on buffers of exactly
their size (tests/native/seq_emu/drive.py).  Bounds are those of oracle/seq.py.  No GPU is involved."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2407_02109_amd", "csrc")
EMU = os.path.join(ROOT, "tests", "native", "host_emu")
SEQ_EMU = os.path.join(ROOT, "tests", "native", "seq_emu")


def _compiler():
    for cand in ("/opt/rocm/llvm/bin/clang++", shutil.which("clang++")):
        if cand and os.path.exists(cand):
            return cand
    return None


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    cxx = _compiler()
    if cxx is None:
        pytest.skip("no clang++ for the host build")
    runtime = subprocess.run([cxx, "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True,
                             text=True).stdout.strip()
    if not os.path.exists(runtime):
        pytest.skip("no shared sanitizer runtime")
    d = tmp_path_factory.mktemp("seq_emu")
    sources = [os.path.join(SEQ_EMU, "emu.cpp")]
    for name in ("fla_seq_api.cpp", "fla_rms_norm.hip", "fla_rotary.hip", "fla_gated_scan.hip"):
        to = d / (name.split(".")[0] + ".cpp")
        shutil.copy(os.path.join(CSRC, name), to)
        sources.append(str(to))
    lib = str(d / "libseq_emu.so")
    cmd = [cxx, "-std=c++20", "-O1", "-g", "-shared", "-fPIC", "-shared-libsan", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", "-fno-sanitize=alignment,vptr,function", "-fno-omit-frame-pointer",
           "-include", os.path.join(SEQ_EMU, "seq_host.h"), "-I", EMU, "-I", CSRC, "-I", os.path.join(ROOT, "include"),
           *sources, "-o", lib]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    if r.returncode != 0:
        pytest.fail("host build failed:\n" + r.stderr[-4000:])
    return lib, runtime


@pytest.mark.parametrize("group", ["norm", "norm_wide", "rotary", "scan"])
def test_kernels_on_the_host(library, group):
    lib, runtime = library
    env = dict(os.environ, LD_PRELOAD=runtime, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:verify_asan_link_order=0:"
                                                                    "detect_stack_use_after_return=0")
    r = subprocess.run([sys.executable, os.path.join(SEQ_EMU, "drive.py"), lib, group], capture_output=True, text=True,
                       timeout=900, env=env)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("ok"), r.stdout[-1500:] + r.stderr[-4000:]
