"""Builds liblcma.so: runs the kernel generator, compiles every translation unit for gfx950
with hipcc and links them.  Usage: python -m paper_2605_06057_amd.build [--force] [-j N]"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys
import time

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
GEN = os.path.join(CSRC, "generated")
LIB = os.path.join(PKG, "liblcma.so")
CALLS = os.path.join(PKG, "_calls.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
DEVICE_FLAGS = ["--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["-O3", "-std=c++17", "-fPIC", "-I", CSRC, "-I", GEN, "-Wno-unused-command-line-argument"]
COMMON += os.environ.get("LCMA_EXTRA_FLAGS", "").split()  # e.g. -D switches of timing experiments


def _newer(target: str, deps: list[str]) -> bool:
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.getmtime(d) <= t for d in deps)


def _compile(src: str, obj: str, deps: list[str], force: bool) -> str:
    if not force and _newer(obj, [src] + deps):
        return f"up to date  {os.path.basename(src)}"
    t0 = time.time()
    flags = COMMON + (DEVICE_FLAGS if src.endswith(".hip") else ["-x", "c++"])
    cmd = [HIPCC] + flags + ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "is not a recognized feature" not in l)
    if r.returncode:
        raise RuntimeError(f"{' '.join(cmd)}\n{err}")
    return f"compiled {time.time() - t0:5.1f}s  {os.path.basename(src)}" + (("\n" + err) if err.strip() else "")


def _calls_built_for() -> str:
    """What _calls.so depends on beside its sources: the interpreter and the torch that it is compiled against ("" without torch)."""
    import importlib.metadata
    import sysconfig
    try:
        return f"{sysconfig.get_config_var('SOABI')} {sys.version_info[:3]} torch {importlib.metadata.version('torch')}"
    except importlib.metadata.PackageNotFoundError:
        return ""


def _calls_missing() -> str:
    """What is not there of the headers that calls.cc needs ("": nothing)."""
    import importlib.util
    import sysconfig
    torch = importlib.util.find_spec("torch")
    if torch is None:
        return "torch"
    if not os.path.exists(os.path.join(os.path.dirname(torch.origin), "include", "torch", "csrc", "autograd", "python_variable.h")):
        return "torch's C++ headers"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    return ""


def _build_calls(force: bool) -> str:
    """_calls.so, the Python side of the calls in csrc/calls.cc, against the torch that is installed and liblcma.so beside it.  liblcma.so needs neither Python nor
    torch: without their headers it is all that is built, and an older _calls.so, which may be another torch's, does not stay."""
    src = os.path.join(CSRC, "calls.cc")
    stamp, built_for = os.path.join(GEN, "calls.built_for"), _calls_built_for()
    if not force and _newer(CALLS, [src, os.path.join(PKG, "..", "include", "lcma.h")]) and os.path.exists(stamp) and open(stamp).read() == built_for:
        return "up to date  calls.cc"
    if os.path.exists(CALLS):
        os.remove(CALLS)
    if missing := _calls_missing():
        return f"not built  calls.cc: {missing} not found; the calls in 8 and 4 bits, the experts' and the tokens' are left out of the Python binding"
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths
    t0 = time.time()
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    rocm = os.path.dirname(os.path.dirname(HIPCC))
    tmp = CALLS + f".tmp{os.getpid()}"
    cmd = [HIPCC, "-x", "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wno-unused-command-line-argument", "-D__HIP_PLATFORM_AMD__=1", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += [f"-I{d}" for d in include_paths() + [sysconfig.get_paths()["include"], os.path.join(rocm, "include")]]
    cmd += [src, "-o", tmp, f"-L{libs}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip", f"-L{PKG}", "-l:liblcma.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError(f"{' '.join(cmd)}\n{r.stderr}")
    os.replace(tmp, CALLS)
    with open(stamp, "w") as f:
        f.write(built_for)
    return f"compiled {time.time() - t0:5.1f}s  calls.cc"


def build(force: bool = False, jobs: int | None = None, verbose: bool = True) -> str:
    from .gen.generate import generate

    hips = generate(GEN)
    headers = [os.path.join(CSRC, h) for h in ("lcma_device.hpp", "lcma_prepare_b.hpp", "lcma_combine_h.hpp", "lcma_params.h", "host_common.h", "lcma_fp8.hpp", "lcma_plane_gemm.hpp", "lcma_pingpong.hpp", "lcma_kpair.hpp", "lcma_pingpong_narrow.hpp", "lcma_few_rows.hpp", "lcma_direct.hpp", "lcma_direct16.hpp", "lcma_i8.hpp", "lcma_i8_pingpong.hpp", "lcma_i8_narrow.hpp", "lcma_i8_few_rows.hpp", "lcma_lanes.hpp", "lcma_experts.hpp", "lcma_experts_ring.hpp", "lcma_experts_pingpong.hpp", "lcma_experts_narrow.hpp", "lcma_experts_any.hpp", "lcma_gated.hpp", "lcma_i4.hpp", "lcma_experts_params.h", "experts_host.h")]
    headers.append(os.path.join(PKG, "..", "include", "lcma.h"))
    headers.append(os.path.join(GEN, "builtin_schemes.inc"))
    units = [(h, h[:-4] + ".o") for h in hips]
    for name in ("api.cc", "scheme.cc", "model.cc", "unfused.cc", "lcma_aux.hip", "lcma_static.hip", "lcma_fp8.hip", "fp8_api.cc", "lcma_plane_gemm.hip", "plane_gemm.cc", "lcma_few_rows.hip", "lcma_small_plain.hip", "lcma_i8.hip", "i8_api.cc", "lcma_tokens.hip", "tokens_api.cc", "lcma_experts.hip", "lcma_gated.hip", "experts_api.cc", "lcma_i4.hip", "i4_api.cc"):
        units.append((os.path.join(CSRC, name), os.path.join(GEN, os.path.splitext(name)[0] + ".o")))
    units.append((os.path.join(GEN, "registry.cc"), os.path.join(GEN, "registry.o")))
    jobs = jobs or min(8, os.cpu_count() or 1)
    with cf.ThreadPoolExecutor(jobs) as ex:
        for msg in ex.map(lambda u: _compile(u[0], u[1], headers, force), units):
            if verbose:
                print(msg, flush=True)
    objs = [o for _, o in units]
    if force or not _newer(LIB, objs):
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.check_call([HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", tmp] + objs)
        os.replace(tmp, LIB)
        if verbose:
            print(f"linked {LIB}", flush=True)
    msg = _build_calls(force)
    if verbose:
        print(msg, flush=True)
    return LIB


if __name__ == "__main__":
    j = None
    if "-j" in sys.argv:
        j = int(sys.argv[sys.argv.index("-j") + 1])
    build(force="--force" in sys.argv, jobs=j)
