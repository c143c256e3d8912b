"""The host code of the row-grouped products, the head's loss and the gradient
clipping (checks of arguments, plans, workspace layout, launches) built for
the CPU with AddressSanitizer and UndefinedBehaviorSanitizer and driven through
thousands of random calls (tests/host_stub/rows_driver.cpp): what every launch
reads and writes has to lie in the call's tensors and in a workspace of the
size that was asked for.  No GPU is needed."""

import concurrent.futures
import hashlib
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
STUB = os.path.join(HERE, "host_stub")
CSRC = os.path.join(ROOT, "paper_2601_13776_amd", "csrc")
BUILD = os.path.join(STUB, "_build")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
UNITS = ["rows.hip", "rows_bf16.hip", "rows_direct.hip", "rows_f32.hip", "rows_few.hip", "grad_clip.hip"]
HEADERS = ["rows.h", "internal.h", "mfma_bf16.h"]
# host-side sanitizer flags (each -fsanitize= after -Xarch_host: host code only)
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
       "-Xarch_host", "-fno-sanitize-recover=undefined"]


def build_driver():
    """Compile (once per source state); returns the driver's path."""
    drv = os.path.join(STUB, "rows_driver.cpp")
    srcs = [os.path.join(CSRC, f) for f in UNITS + HEADERS] + [os.path.join(ROOT, "include", "orth.h"), drv]
    h = hashlib.sha256()
    for f in srcs:
        h.update(open(f, "rb").read())
    tag = h.hexdigest()[:16]
    exe = os.path.join(BUILD, f"rows_driver_{tag}")
    if os.path.exists(exe):
        return exe
    os.makedirs(BUILD, exist_ok=True)

    def compile(src):
        obj = os.path.join(BUILD, f"{tag}_{os.path.basename(src)}.o")
        r = subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-g", "-std=c++17", "-fPIC", *SAN,
                            "-Wno-unused-command-line-argument", "-c", src, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        return obj

    with concurrent.futures.ThreadPoolExecutor(4) as pool:
        objs = list(pool.map(compile, [os.path.join(CSRC, f) for f in UNITS] + [drv]))
    # (the device code, which is not there, is an address only)
    r = subprocess.run(["/opt/rocm/llvm/bin/clang++", "-fsanitize=address", "-fsanitize=undefined",
                        "-Wl,--unresolved-symbols=ignore-in-object-files", *objs, "-o", exe + ".tmp"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    os.replace(exe + ".tmp", exe)
    return exe


def run(*args):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    return subprocess.run([build_driver(), *args], capture_output=True, text=True, env=env, timeout=600)


@pytest.mark.slow
def test_launches_stay_in_the_calls_memory():
    r = run()
    assert r.returncode == 0 and r.stdout.startswith("calls "), r.stdout[-500:] + r.stderr[-3000:]


@pytest.mark.slow
def test_a_short_workspace_is_seen():
    """Workspaces declared 256 bytes shorter than was asked for: some call fills
    its last bytes."""
    r = run("256")
    assert r.returncode == 3 and "outside the call's memory" in r.stderr, r.stderr[-500:]
