"""Builds libmuon_mi355x.so (the optimizer), libmuon_layers.so (the layer
operators), libmuon_adamw.so (the AdamW step), and libmuon_diag.so (a matrix-core
ceiling probe the bench reports as context) for gfx950 with hipcc, and the extensions
that read torch's tensors for the layer operators and AdamW with the host's compiler;
in-tree, no JIT cache.

Usage: python -m paper_2606_27153_amd.build [-v]
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB_NAME = "libmuon_mi355x.so"
LIB_PATH = os.path.join(PKG, LIB_NAME)
ARCH = "gfx950"

# the GEMM kernels are instantiated in several translation units (the 256
# tile's B*X and square-output kernels per operand type, the smaller tiles)
# so that they compile in parallel
SOURCES = ["api.cpp", "plan.cpp", "ew_kernels.hip", "ns_gemm.hip", "ns_gemm_t256_bf16_bx.hip",
           "ns_gemm_t256_bf16_sq.hip", "ns_gemm_t256_f16_bx.hip", "ns_gemm_t256_f16_sq.hip", "ns_tile_bf16.hip",
           "ns_tile_f16.hip", "ns_tile_f32.hip", "static_ws.hip"]
LAYER_SOURCES = ["layers/layers_api.cpp", "layers/mm_simple.hip", "layers/mm_tile_256_bf16.hip",
                 "layers/mm_tile_128x256_bf16.hip", "layers/mm_tile_128_bf16.hip", "layers/mm_tile_128_f32.hip",
                 "layers/mm_tile_64_bf16.hip", "layers/mm_tile_64_f32.hip", "layers/mm_skinny.hip",
                 "layers/pack.hip", "layers/act_grad.hip", "layers/layer_norm.hip",
                 "layers/tokens_api.cpp", "layers/routing.hip", "layers/embedding.hip", "layers/loss.hip",
                 "layers/mm_loss_256_bf16.hip", "layers/mm_loss_128x256_bf16.hip", "layers/mm_loss_128_bf16.hip",
                 "layers/mm_loss_64_bf16.hip", "layers/mm_loss_128_f32.hip", "layers/mm_loss_64_f32.hip"]
ADAMW_SOURCES = ["adamw/adamw_api.cpp", "adamw/adamw.hip"]
ADAMW_LIB_PATH = os.path.join(PKG, "libmuon_adamw.so")
LAYER_LIB_PATH = os.path.join(PKG, "libmuon_layers.so")
# CPython extensions that read torch's tensors (host code): source, path, and the library they call
BINDINGS = [("adamw/binding.cpp", os.path.join(PKG, "_adamw_binding.so"), None),
            ("layers/binding.cpp", os.path.join(PKG, "_layers_binding.so"), "muon_layers")]
DIAG_SOURCES = ["diag/mfma_ceiling.hip"]
DIAG_LIB_PATH = os.path.join(PKG, "libmuon_diag.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

COMMON = [
    "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
    f"--offload-arch={ARCH}",
    # no packed fp32 instructions in any device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # keep per-thread staging arrays in registers, never in LDS
    "-mllvm", "-disable-promote-alloca-to-lds",
    "-I" + os.path.join(ROOT, "include"),
    "-Wall", "-Wno-unused-result",
]


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [HIPCC, *COMMON, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops' is not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{out}")
    if verbose and out.strip():
        print(out)
    return obj


def _link(objs, path: str, verbose: bool) -> None:
    tmp = path + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, path)


def _run(cmd, what: str, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"building {what} failed:\n{r.stdout}{r.stderr}")


def _compile_binding(src: str, verbose: bool) -> str:
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    obj = os.path.join(BUILD, src.replace("/", "_") + ".o")
    _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-D__HIP_PLATFORM_AMD__",
          "-I" + os.path.join(ROOT, "include"), *("-isystem" + d for d in cpp_extension.include_paths()),
          "-isystem" + sysconfig.get_paths()["include"], "-c", os.path.join(CSRC, src), "-o", obj], src, verbose)
    return obj


def _link_binding(obj: str, path: str, library, verbose: bool) -> None:
    import torch
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    own = [f"-L{PKG}", f"-l{library}", "-Wl,-rpath,$ORIGIN"] if library else []
    _run([os.environ.get("CXX", "g++"), "-shared", obj, "-o", path + ".tmp", *own, "-L" + lib, "-ltorch_python",
          "-ltorch_cpu", "-lc10", "-Wl,-rpath," + lib], path, verbose)
    os.replace(path + ".tmp", path)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    parts = ((SOURCES, LIB_PATH), (LAYER_SOURCES, LAYER_LIB_PATH), (ADAMW_SOURCES, ADAMW_LIB_PATH),
             (DIAG_SOURCES, DIAG_LIB_PATH))
    srcs = [s for sources, _ in parts for s in sources]
    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 4)) as ex:
        bindings = [ex.submit(_compile_binding, src, verbose) for src, _, _ in BINDINGS]
        objs = dict(zip(srcs, ex.map(lambda s: _compile(s, verbose), srcs)))
        bindings = [b.result() for b in bindings]
    for sources, path in parts:
        _link([objs[s] for s in sources], path, verbose)
    for obj, (_, path, library) in zip(bindings, BINDINGS):
        _link_binding(obj, path, library, verbose)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
