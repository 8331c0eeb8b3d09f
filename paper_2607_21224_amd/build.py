"""Build the gfx950 shared library of the CPDP path (and the synthetic-input
library the tests and benchmark use) with hipcc, in-tree."""
from __future__ import annotations

import os
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

LIB_CPDP = os.path.join(PKG, "libcpdp.so")
# the same sources with 256-thread blocks: a different launch shape for the
# tests that check results do not depend on it
LIB_CPDP_BLOCK256 = os.path.join(PKG, "libcpdp_block256.so")
# the 8-bit activation path (include/cpdp_q8.h)
LIB_Q8 = os.path.join(PKG, "libcpdp_q8.so")
# its Python extension (host code)
EXT_Q8 = os.path.join(PKG, "_q8" + sysconfig.get_config_var("EXT_SUFFIX"))
LIB_SYNTH = os.path.join(ROOT, "synth", "libsynth.so")

# -ffp-contract=off: only the explicit fmaf calls fuse, so the arithmetic is
# exactly what the source says.  Packed fp32 instructions are disabled.
COMPILE_FLAGS = [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
                 "-ffp-contract=off", "-Xclang", "-target-feature", "-Xclang",
                 "-packed-fp32-ops", "-Wall", "-Wno-unused-command-line-argument"]
HIP_FLAGS = COMPILE_FLAGS + ["-shared"]

# the kernel translation units of libcpdp.so (compiled in parallel) and the
# host validation layer
KERNEL_SOURCES = ("kernels_flat.hip", "kernels_sync_cpdp.hip", "kernels_sync_localsgd.hip",
                  "kernels_sync_ddp.hip", "kernels_plan.hip", "kernels_plan_table.hip",
                  "kernels_table.hip", "kernels_check.hip")
# headers the kernel sources include (part of what the recorded traffic is for)
KERNEL_HEADERS = ("cpdp_device.h", "cpdp_sync_impl.h", "cpdp_split.h", "cpdp_dispatch.h",
                  "cpdp_plan_impl.h", "cpdp_launch.h")
HOST_SOURCES = ("cpdp_api.cpp",)
# the library's own device memory (no kernels): the static plan table
SCRATCH_SOURCES = ("plan_scratch.hip",)
# gradient norms and clipping (part of libcpdp.so; no kernel of a step)
CLIP_SOURCES = ("kernels_clip.hip", "clip_api.cpp")
# libcpdp_q8.so: kernel translation units and the host validation layer
Q8_SOURCES = ("q8_rows.hip", "q8_norm.hip", "q8_act.hip", "q8_matmul.hip", "q8_grad.hip",
              "q8_grad_few.hip", "q8_api.cpp")
# the loss on that path (in the same library)
XENT_SOURCES = ("q8_xent.hip", "q8_xent_few.hip", "q8_xent_api.cpp")
OBJ_ROOT = os.path.join(ROOT, "_build")


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("build failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)


def build_cpdp(out: str = LIB_CPDP, extra=(),
               sources=KERNEL_SOURCES + HOST_SOURCES + SCRATCH_SOURCES + CLIP_SOURCES) -> str:
    from concurrent.futures import ThreadPoolExecutor
    csrc = os.path.join(PKG, "csrc")
    objdir = os.path.join(OBJ_ROOT, os.path.basename(out) + ".objs")
    os.makedirs(objdir, exist_ok=True)

    def compile_one(name):
        obj = os.path.join(objdir, name + ".o")
        _run([HIPCC, *COMPILE_FLAGS, *extra, "-I", os.path.join(ROOT, "include"), "-I", csrc,
              "-c", "-o", obj, os.path.join(csrc, name)])
        return obj

    with ThreadPoolExecutor(len(sources)) as ex:
        objs = list(ex.map(compile_one, sources))
    tmp = out + ".tmp"
    _run([HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs])
    os.replace(tmp, out)
    return out


def build_q8(out: str = LIB_Q8) -> str:
    return build_cpdp(out, sources=Q8_SOURCES + XENT_SOURCES)


def build_q8_extension(out: str = EXT_Q8) -> str:
    """The Python extension that marshals the 8-bit path's arguments, linked to
    libcpdp_q8.so beside it and to the torch libraries that torch has loaded."""
    import torch
    root = os.path.dirname(torch.__file__)
    tmp = out + ".tmp"
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-fvisibility=hidden",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
          "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
          "-I", sysconfig.get_paths()["include"], "-isystem", os.path.join(root, "include"),
          "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
          "-isystem", os.path.join(os.path.dirname(os.path.dirname(HIPCC)), "include"),
          "-o", tmp, os.path.join(PKG, "csrc", "q8_bind.cpp"), "-L", PKG, "-lcpdp_q8",
          "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip",
          "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, out)
    return out


def build_synth(out: str = LIB_SYNTH) -> str:
    tmp = out + ".tmp"
    _run([HIPCC, *HIP_FLAGS, "-o", tmp, os.path.join(ROOT, "synth", "synth.hip")])
    os.replace(tmp, out)
    return out


CONSUMER = os.path.join(ROOT, "tests", "consumer", "abi_consumer")


def build_consumer(out: str = CONSUMER) -> str:
    """The torch-free host program of the ABI tests, linked to libcpdp.so."""
    tmp = out + ".tmp"
    _run([HIPCC, "-O2", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "include"),
          "-o", tmp, out + ".cpp", "-L", PKG, "-lcpdp",
          "-Wl,-rpath,$ORIGIN/../../paper_2607_21224_amd"])
    os.replace(tmp, out)
    return out


def build_all() -> None:
    from concurrent.futures import ThreadPoolExecutor
    with ThreadPoolExecutor(4) as ex:
        jobs = [ex.submit(build_cpdp), ex.submit(build_q8), ex.submit(build_synth),
                ex.submit(build_cpdp, LIB_CPDP_BLOCK256, ("-DCPDP_BLOCK=256",))]
        for j in jobs:
            j.result()
    build_consumer()
    build_q8_extension()


if __name__ == "__main__":
    build_all()
    print("built", LIB_CPDP, LIB_SYNTH)
