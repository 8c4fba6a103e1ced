"""Build libtq.so (the HIP kernels and the C ABI) in place for gfx950, and, where a PyTorch
for ROCm is installed, _tqtorch.so (the native half of kvcache.py, against it)."""
import glob
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libtq.so")
BINDING = os.path.join(HERE, "_tqtorch.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# any C++ compiler for the host: without g++ the one that comes with hipcc
CXX = os.environ.get("CXX") or shutil.which("g++") or os.path.join(os.path.dirname(HIPCC), "amdclang++")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # packed fp32 VALU instructions are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # matrix-core results land in VGPRs (no accumulator-register copies)
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    "-Wall", "-Wno-unused-function",
    "-parallel-jobs=8",            # the files beside each other
]


def sources():
    return sorted(glob.glob(os.path.join(HERE, "csrc", "*.hip")))


def build(verbose: bool = False) -> str:
    cmd = [HIPCC, *FLAGS, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc"),
           *sources(), "-o", LIB + ".tmp"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(LIB + ".tmp", LIB)
    if has_torch():
        build_binding(verbose)
    else:
        print("no PyTorch for ROCm here: libtq.so only, without _tqtorch.so", flush=True)
    return LIB


def has_torch() -> bool:
    """Whether the binding has something to be built against (the C library needs none)."""
    try:
        import torch
    except ImportError:
        return False
    return torch.version.hip is not None


def build_binding(verbose: bool = False) -> str:
    import torch
    t = os.path.dirname(torch.__file__)
    cmd = [CXX, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(x for d in (os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"),
                         sysconfig.get_paths()["include"]) for x in ("-isystem", d)),
           "-I", os.path.join(ROOT, "include"), os.path.join(HERE, "csrc", "tq_torch.cpp"), "-o", BINDING + ".tmp",
           "-L", os.path.join(t, "lib"), "-ltorch_python", "-ltorch", "-ltorch_hip", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(BINDING + ".tmp", BINDING)
    return BINDING


if __name__ == "__main__":
    build(verbose=True)
