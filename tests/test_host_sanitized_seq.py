"""The sequence operators' entry points (seq.hip: argument checks, offset arithmetic) under AddressSanitizer and
UndefinedBehaviorSanitizer, host side only: tests/test_seq_abi.py runs against a library with that one source
instrumented (each -fsanitize= behind -Xarch_host, the device code untouched).  CPU only."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OUT = os.path.join(ROOT, "_build", "asan")
HOST_SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
            "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
CHILD = r"""
import sys
sys.path.insert(0, {root!r})
from paper_2103_08802_amd import binding as B
B.LIB_PATH = {lib!r}
import pytest
rc = pytest.main(["-q", "-x", "-s", "-p", "no:cacheprovider", {tests!r}])
assert B.lib()._name == {lib!r}
sys.exit(rc)
"""


def test_seq_abi_under_asan_and_ubsan():
    r = subprocess.run(["hipcc", "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True)
    rt = r.stdout.strip()
    if r.returncode != 0 or not os.path.isabs(rt) or not os.path.exists(rt):
        pytest.skip("no ASan runtime in this toolchain")
    sys.path.insert(0, ROOT)
    import __graft_entry__ as G
    os.makedirs(OUT, exist_ok=True)
    objs = []
    for src in G.SOURCES:                      # the ordinary objects of the last build, else compile
        if src == "seq.hip":
            continue
        obj = os.path.join(G.BUILD, os.path.splitext(src)[0] + ".o")
        objs.append(obj if os.path.exists(obj) else G._compile(src))
    seq = os.path.join(OUT, "seq.o")
    r = subprocess.run(["hipcc"] + [f for f in G.HIPCC_FLAGS if f != "-O3"] + ["-O1", "-g"] + HOST_SAN +
                       ["-c", os.path.join(G.CSRC, "seq.hip"), "-o", seq], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    lib = os.path.join(OUT, "libpnn_asan_seq.so")
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", lib, seq] + objs,
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ)
    env["LD_PRELOAD"] = rt + (":" + env["LD_PRELOAD"] if env.get("LD_PRELOAD") else "")
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=1"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1"
    code = CHILD.format(root=ROOT, lib=lib, tests=os.path.join(ROOT, "tests", "test_seq_abi.py"))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, env=env, timeout=600)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert r.returncode == 0, out[-6000:]
    assert " passed" in out
