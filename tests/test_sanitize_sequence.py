"""The sequence operators' host code under AddressSanitizer and
UndefinedBehaviorSanitizer (runs without a GPU): tests/sanitize/sequence_fuzz.c
against a build of the two host files whose host pass is instrumented."""
import importlib.util
import os
import subprocess

import pytest

from conftest import ROOT


def _build():
    path = os.path.join(ROOT, "tests", "sanitize", "build.py")
    spec = importlib.util.spec_from_file_location("sanitize_build", path)
    base = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(base)
    lb = base.libbuild
    exe, lib = os.path.join(base.OUT, "sequence_fuzz"), os.path.join(base.OUT, "libmdlstm_sequence_san.so")
    if os.path.exists(exe) and os.path.getmtime(exe) >= os.path.getmtime(lb.LIB):
        return exe
    os.makedirs(base.OUT, exist_ok=True)
    kernels = [os.path.join(lb.BUILD, os.path.splitext(s)[0] + ".o") for s in lb.SOURCES if s.endswith(".hip")]
    missing = [k for k in kernels if not os.path.exists(k)]
    if missing:
        raise RuntimeError(f"regular build objects missing: {missing}")
    host_san = [x for f in base.SAN for x in ("-Xarch_host", f)]
    objs = []
    for src in (s for s in lb.SOURCES if s.endswith(".cpp")):
        objs.append(os.path.join(base.OUT, "sequence_" + os.path.splitext(src)[0] + ".o"))
        base._run([lb.HIPCC, *lb.FLAGS, "-O1", "-g", *host_san, "-x", "hip", "-c", os.path.join(lb.CSRC, src), "-o", objs[-1]])
    base._run([lb.HIPCC, f"--offload-arch={lb.ARCH}", "-shared", "-fPIC", *host_san, *objs, *kernels, "-o", lib])
    base._run([base.CLANG, "-std=c11", "-O1", "-g", *base.SAN, "-I", lb.INCLUDE,
               os.path.join(ROOT, "tests", "sanitize", "sequence_fuzz.c"), "-o", exe, lib, "-lm", f"-Wl,-rpath,{base.OUT}"])
    return exe


def test_sequence_host_checks_under_sanitizers(built_lib):
    try:
        exe = _build()
    except RuntimeError as e:
        pytest.skip(f"sanitizer build unavailable: {e}")
    env = dict(os.environ)
    env.update(HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="", CUDA_VISIBLE_DEVICES="",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe, "20000"], capture_output=True, text=True, env=env, timeout=300)
    out = r.stdout + r.stderr
    print(r.stdout)
    assert r.returncode == 0, out[-4000:]
    assert "runtime error" not in out and "AddressSanitizer" not in out, out[-4000:]
    assert " 0 failures" in r.stdout
