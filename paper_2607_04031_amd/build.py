"""Build libtl.so (HIP kernels + C ABI) in-tree for gfx950 with hipcc, and
_tl_torch.so (host code that takes torch tensors to it) with the C++ compiler.

    python -m paper_2607_04031_amd.build          # or build() from Python
"""
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtl.so")
CALLS = os.path.join(HERE, "_tl_torch.so")
SOURCES = ["tl_api.cpp", "tl_read_amp.cpp", "tl_view.cpp", "tl_repack.hip", "tl_decode.hip", "tl_decode_fp8.hip",
           "tl_decode_lds.hip", "tl_lgms.hip", "tl_prefill.hip", "tl_view.hip", "tl_stream.hip",
           "tl_scratch.hip", "tl_decode_kn.hip", "tl_medium.hip", "tl_serve.cpp", "tl_kv.hip", "tl_attn.hip",
           "tl_attn_wide.hip", "tl_verify.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    "-Wall",
    # packed fp32 VALU ops are kept out of the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + os.path.join(ROOT, "include"),
]


def calls_command(out: str) -> list:
    """Compiles the extension module over libtl; libtl is found beside it."""
    import torch
    home = os.path.dirname(torch.__file__)
    # HIPCC may be a name that PATH finds, or a link into the installation
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which(HIPCC) or HIPCC)))
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
            "-DUSE_ROCM=1", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-isystem", os.path.join(home, "include"), "-isystem", os.path.join(rocm, "include"),
            "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "tl_torch.cpp"), "-o", out,
            "-L" + os.path.join(home, "lib"), "-ltorch_python", "-lc10_hip", "-lc10", "-ltorch_cpu",
            "-L" + HERE, "-l:libtl.so", "-Wl,-rpath,$ORIGIN"]


def build(verbose: bool = False, jobs: int = 8) -> str:
    """Compile every source to an object in parallel, then link libtl.so."""
    objdir = os.path.join(ROOT, "_build", "libtl")
    os.makedirs(objdir, exist_ok=True)
    procs, objs = [], []
    for src in SOURCES:
        obj = os.path.join(objdir, src + ".o")
        objs.append(obj)
        lang = ["-x", "hip"] if src.endswith(".hip") else []
        cmd = [HIPCC] + [f for f in FLAGS if f != "-shared"] + ["-c"] + lang + [os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        text = out.decode(errors="replace")
        # the host pass does not know the device-only feature flag; that note is harmless
        lines = [l for l in text.splitlines() if "packed-fp32-ops" not in l and l.strip()]
        if p.returncode != 0:
            failed.append(src)
            print("\n".join(lines), file=sys.stderr)
        elif verbose and lines:
            print("\n".join(lines))
    if failed:
        raise RuntimeError("hipcc failed for: " + ", ".join(failed))
    link = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC"] + objs + ["-o", LIB + ".tmp"]
    if verbose:
        print(" ".join(link), flush=True)
    subprocess.run(link, check=True)
    os.replace(LIB + ".tmp", LIB)
    if verbose:
        print(" ".join(calls_command(CALLS)), flush=True)
    subprocess.run(calls_command(CALLS + ".tmp"), check=True)
    os.replace(CALLS + ".tmp", CALLS)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
