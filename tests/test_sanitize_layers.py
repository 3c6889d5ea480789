"""The host code of the gated recurrence, the group norm and the loss over a vocabulary
under AddressSanitizer and UndefinedBehaviorSanitizer (runs without a GPU):
tests/sanitize/layers_fuzz.c against the library whose host files are instrumented."""
import os
import subprocess

import pytest

import test_sanitize_sequence as sequence
from conftest import ROOT


def _build():
    lib = os.path.join(os.path.dirname(sequence._build()), "libmdlstm_sequence_san.so")
    out, source = os.path.join(os.path.dirname(lib), "layers_fuzz"), os.path.join(ROOT, "tests", "sanitize", "layers_fuzz.c")
    spec = sequence.importlib.util.spec_from_file_location("sanitize_build", os.path.join(ROOT, "tests", "sanitize", "build.py"))
    base = sequence.importlib.util.module_from_spec(spec)
    spec.loader.exec_module(base)
    if not os.path.exists(out) or os.path.getmtime(out) < max(os.path.getmtime(lib), os.path.getmtime(source)):
        base._run([base.CLANG, "-std=c11", "-O1", "-g", *base.SAN, "-I", base.libbuild.INCLUDE, source, "-o", out, lib,
                   f"-Wl,-rpath,{os.path.dirname(lib)}"])
    return out


def test_layers_host_checks_under_sanitizers(built_lib):
    try:
        exe = _build()
    except RuntimeError as e:
        pytest.skip(f"sanitizer build unavailable: {e}")
    env = dict(os.environ)
    env.update(HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="", CUDA_VISIBLE_DEVICES="",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe, "5000"], capture_output=True, text=True, env=env, timeout=300)
    out = r.stdout + r.stderr
    print(r.stdout)
    assert r.returncode == 0, out[-4000:]
    assert "runtime error" not in out and "AddressSanitizer" not in out, out[-4000:]
    assert " 0 failures" in r.stdout
