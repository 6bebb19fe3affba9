"""AddressSanitizer and UndefinedBehaviorSanitizer over the host side of the
gated block, the residual norms and AdamW with 8-bit states: argument checks
(train_ops.cpp) and launchers are compiled again with both sanitizers on their
host code only and run by host_sanitize_blocks_driver.cpp with every launch
skipped, so no GPU is needed.  Needs the in-tree build (the other kernels'
objects) and hipcc."""
import concurrent.futures
import glob
import os
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2004_09910_amd")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CLANG = "/opt/rocm/llvm/bin/clang++"
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
       "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
SOURCES = ["runtime.cpp", "prof.cpp", "train_ops.cpp", "gated.hip", "residual_norm.hip", "adamw8.hip"]


def _run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert r.returncode == 0, f"{' '.join(cmd)}\n{r.stdout[-3000:]}\n{r.stderr[-3000:]}"
    return r


def test_host_side_of_block_operators_under_asan_and_ubsan():
    kernels = [k for k in sorted(glob.glob(os.path.join(PKG, "_build", "*.hip.o")))
               if os.path.basename(k)[:-2] not in SOURCES]
    if not (os.path.exists(HIPCC) and os.path.exists(CLANG) and kernels):
        pytest.skip("needs hipcc, clang++ and the in-tree build's kernel objects")
    inc = ["-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(PKG, "csrc")]
    with tempfile.TemporaryDirectory() as tmp:
        def compile_(src):
            o = os.path.join(tmp, src + ".o")
            _run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC",
                  "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"] + SAN + inc +
                 ["-c", os.path.join(PKG, "csrc", src), "-o", o])
            return o

        with concurrent.futures.ThreadPoolExecutor(4) as pool:
            objs = list(pool.map(compile_, SOURCES))
        exe = os.path.join(tmp, "driver")
        _run([CLANG, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined",
              "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer"] + inc +
             [os.path.join(ROOT, "tests", "host_sanitize_blocks_driver.cpp")] + objs + kernels +
             ["-L/opt/rocm/lib", "-lamdhip64", "-lrocprofiler-sdk-roctx",
              "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
        env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
                   UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
        r = _run([exe], env=env, timeout=300)
        assert "host operators: ok" in r.stdout
