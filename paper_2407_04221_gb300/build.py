"""Compile libautoverse.so in-tree for sm_103a (nvcc, no cmake) and the policy
operators' binding, _policy.so (g++, against the installed torch)."""
from __future__ import annotations

import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libautoverse.so")
SOURCES = [os.path.join(CSRC, f) for f in ("autoverse.cu", "k_fast_u8.cu", "k_fast_u16.cu", "k_warp_u8.cu",
                                            "k_warp_u16.cu", "k_block.cu", "k_expand.cu", "k_search.cu",
                                            "k_observe.cu", "k_mutate.cu", "k_memo_u8.cu", "k_memo_u16.cu",
                                            "k_vmemo_u8.cu", "k_vmemo_u16.cu", "k_vmany_u8.cu", "k_vmany_u16.cu",
                                            "k_variant.cu", "k_band.cu", "k_step.cu", "policy.cu", "k_norm.cu",
                                            "k_scan.cu", "k_logp.cu", "k_ffn.cu")]
DEPS = SOURCES + [os.path.join(CSRC, f) for f in ("kernels.cuh", "launch.h", "k_fast_impl.cuh", "k_warp_impl.cuh",
                                                     "k_memo_impl.cuh", "block_step.cuh", "small_step.cuh",
                                                     "variant_keys.cuh", "policy.h", "values.cuh",
                                                     "async.cuh", "tensor_map.h")] + [
    os.path.join(ROOT, "include", "autoverse.h")]
BINDING = os.path.join(CSRC, "policy_binding.cpp")
BINDING_LIB = os.path.join(PKG, "_policy.so")
BINDING_STAMP = os.path.join(PKG, "_build", "policy_torch.txt")  # what it was made for
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _compile_binding(obj: str) -> list:
    """The command that compiles the binding."""
    import sysconfig

    import torch
    at = os.path.dirname(os.path.abspath(torch.__file__))
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    inc = [os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"),
           os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-w", f"-D_GLIBCXX_USE_CXX11_ABI={abi}",
            "-I", os.path.join(ROOT, "include"), *(x for d in inc for x in ("-isystem", d)), "-c", BINDING, "-o", obj]


def _link_binding(obj: str, out: str) -> list:
    import torch
    libs = os.path.join(os.path.dirname(os.path.abspath(torch.__file__)), "lib")
    return ["g++", "-shared", obj, "-o", out, "-L", PKG, "-l:libautoverse.so", "-L", libs, "-ltorch_python",
            "-ltorch_cuda", "-ltorch_cpu", "-ltorch", "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{libs}"]


def _torch_stamp():
    """Which torch the binding is made for; None without one."""
    try:
        import torch
    except ImportError:
        return None
    return f"{torch.__version__} {os.path.abspath(torch.__file__)}\n"


def _read(path):
    try:
        with open(path) as f:
            return f.read()
    except OSError:
        return None


def build(force: bool = False, verbose: bool = False, extra: list | None = None) -> str:
    """Build the shared library and the binding next to this file: every
    translation unit is compiled in parallel, then linked, the library first.
    Without torch the library alone.  Returns the library's path."""
    def stale(lib, deps):
        return not os.path.exists(lib) or any(os.path.getmtime(d) > os.path.getmtime(lib) for d in deps)

    native = bool(force or extra) or stale(LIB, DEPS)
    stamp = _torch_stamp()
    binding = stamp is not None and (native or stale(BINDING_LIB, [BINDING, LIB]) or _read(BINDING_STAMP) != stamp)
    if not (native or binding):
        return LIB
    import tempfile
    from concurrent.futures import ThreadPoolExecutor

    def run(cmd):
        if verbose:
            print(" ".join(cmd))
        subprocess.check_call(cmd)

    cuda_lib = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "lib64")
    common = [nvcc(), "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-lineinfo", *ARCH,
              "-I", os.path.join(ROOT, "include"), *(extra or [])]
    with tempfile.TemporaryDirectory() as tmpdir, ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as pool:
        sources = SOURCES if native else []
        objs = [os.path.join(tmpdir, os.path.basename(src) + ".o") for src in sources]
        glue = os.path.join(tmpdir, "policy_binding.o")
        units = [pool.submit(run, common + ["-c", src, "-o", obj]) for src, obj in zip(sources, objs)]
        bound = pool.submit(lambda: run(_compile_binding(glue))) if binding else None
        for unit in units:
            unit.result()
        if native:
            tmp = LIB + f".tmp{os.getpid()}"
            run([nvcc(), "-shared", *ARCH, "-cudart", "shared", "-Xlinker", "-rpath", "-Xlinker", cuda_lib,
                 "-Xlinker", "-soname", "-Xlinker", os.path.basename(LIB), *objs, "-o", tmp])
            os.replace(tmp, LIB)
        if bound:
            bound.result()
            tmp = BINDING_LIB + f".tmp{os.getpid()}"
            run(_link_binding(glue, tmp))
            os.replace(tmp, BINDING_LIB)
            os.makedirs(os.path.dirname(BINDING_STAMP), exist_ok=True)
            with open(BINDING_STAMP, "w") as f:
                f.write(stamp)
        elif stamp is None:
            print(f"no torch: {os.path.basename(BINDING_LIB)} is not built")
    return LIB


if __name__ == "__main__":
    build(force=True, verbose=True)
