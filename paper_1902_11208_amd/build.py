"""Build libmdlstm.so (the C-ABI library and its HIP kernels) for gfx950, in-tree.

The sequence operators' Python binding (_binding.so, csrc/binding.cpp) is built
beside it with the host compiler against torch's headers.

Usage: python -m paper_1902_11208_amd.build [--verbose]
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libmdlstm.so")
BINDING = os.path.join(PKG, "_binding.so")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", "g++")
ARCH = "gfx950"

SOURCES = ["mdlstm_api.cpp", "k_pack.hip", "k_proj.hip", "k_wave.hip", "k_wave_fwd_f32_h4.hip", "k_wave_fwd_f32_h8.hip",
           "k_wave_fwd_f32_h16.hip", "k_wave_fwd_f32_h32.hip", "k_wave_fwd_f32_h64.hip", "k_wave_fwd_bf16_h32.hip",
           "k_wave_fwd_bf16_h64.hip", "k_wave_bwd_f32_h4.hip", "k_wave_bwd_f32_h8.hip", "k_wave_bwd_f32_h16.hip",
           "k_wave_bwd_f32_h32.hip", "k_wave_bwd_f32_h64.hip", "k_wave_bwd_bf16_h32.hip", "k_wave_bwd_bf16_h64.hip", "k_bwd_big.hip", "k_bwd_strip.hip",
           "k_stack.hip", "k_head.hip", "k_wave_mem_h16.hip", "k_wave_mem_h32.hip", "k_pad.hip",
           "sequence_api.cpp", "k_attention.hip", "k_norm.hip", "layers_api.cpp", "k_recurrence.hip", "k_groupnorm.hip",
           "k_vocabulary.hip"]

FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-fPIC",
    "-std=c++17",
    "-I", INCLUDE,
    "-I", CSRC,
    # packed fp32 VALU ops stay off; the compiler otherwise forms them from scalar code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS]
    if src.endswith(".cpp"):
        cmd += ["-x", "hip"]
    cmd += ["-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        cmd += ["-Rpass-analysis=kernel-resource-usage"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(ln for ln in (r.stdout + r.stderr).splitlines()
                    if "not a recognized feature" not in ln)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{out}")
    if verbose and out.strip():
        print(out)
    return obj


def _compile_binding() -> str:
    import torch

    obj, t = os.path.join(BUILD, "binding.o"), os.path.dirname(torch.__file__)
    abi = int(torch.compiled_with_cxx11_abi())  # std::string as torch's own libraries have it
    includes = [os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(ROCM, "include")]
    cmd = [CXX, "-O2", "-fPIC", "-std=c++17", "-DTORCH_EXTENSION_NAME=_binding", f"-D_GLIBCXX_USE_CXX11_ABI={abi}", "-DUSE_ROCM",
           "-D__HIP_PLATFORM_AMD__", "-I", INCLUDE, *[x for i in includes for x in ("-isystem", i)], "-c",
           os.path.join(CSRC, "binding.cpp"), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{CXX} failed on binding.cpp:\n{r.stdout}\n{r.stderr}")
    return obj


def _link_binding(obj: str) -> None:
    import torch

    tmp = BINDING + ".tmp"
    cmd = [CXX, "-shared", obj, "-o", tmp, "-L", os.path.join(os.path.dirname(torch.__file__), "lib"), "-ltorch_python",
           "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_hip", "-L", PKG, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link of the binding failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BINDING)


def build(verbose: bool = False) -> str:
    """The library, then the binding: the error of a binding that does not build is raised when the library is in
    place, with no binding of an earlier build beside it."""
    os.makedirs(BUILD, exist_ok=True)
    jobs = min(len(SOURCES) + 1, max(1, min(16, os.cpu_count() or 1)))
    with cf.ThreadPoolExecutor(jobs) as ex:
        binding = ex.submit(_compile_binding)
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-Wl,--no-undefined", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    try:
        _link_binding(binding.result())
    except Exception as e:
        if os.path.exists(BINDING):
            os.remove(BINDING)
        raise RuntimeError("libmdlstm.so is built, the sequence operators' binding is not") from e
    return LIB


if __name__ == "__main__":
    print(build(verbose="--verbose" in sys.argv))
