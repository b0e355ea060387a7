"""Build libsmol.so (HIP, gfx950) in-tree with hipcc.

Usage: python -m paper_2007_13005_amd.build [-v]
"""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys
import sysconfig
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libsmol.so")
# the binding's native marshalling, named for this interpreter's ABI
PYCALL = os.path.join(PKG, "_smolcall" + sysconfig.get_config_var("EXT_SUFFIX"))
# the token operators' binding, which reads torch's tensors
PYTOKENS = os.path.join(PKG, "_smoltokens" + sysconfig.get_config_var("EXT_SUFFIX"))

# The row-streaming kernels are split into parts (input, output type, row
# walk, output layout) so that the compiler runs on the parts in parallel.
SOURCES = [
    "smol_kernels.hip",
    "smol_rows_rgb_f16_range.hip",
    "smol_rows_rgb_f16_range_nhwc.hip",
    "smol_rows_rgb_f16_stride.hip",
    "smol_rows_rgb_f16_stride_nhwc.hip",
    "smol_rows_rgb_f32_range.hip",
    "smol_rows_rgb_f32_range_nhwc.hip",
    "smol_rows_rgb_f32_stride.hip",
    "smol_rows_rgb_f32_stride_nhwc.hip",
    "smol_rows_rgb_u8_range.hip",
    "smol_rows_rgb_u8_range_nhwc.hip",
    "smol_rows_yuv_range.hip",
    "smol_rows_yuv_range_nhwc.hip",
    "smol_host.cpp",
    "smol_pipeline.cpp",
    "smol_jpeg_kernels.hip",
    "smol_jpeg.cpp",
    "smol_jpeg_entropy.cpp",
    "smol_stream.hip",
    "smol_scratch.hip",
    "smol_patch.hip",
    "smol_patch_f32.hip",
    "smol_patch_f16.hip",
    "smol_patch_bf16.hip",
    "smol_patch_grad_f32.hip",
    "smol_patch_grad_f16.hip",
    "smol_patch_grad_bf16.hip",
    "smol_embed.hip",
    "smol_norm.hip",
]
HEADERS = ["smol_internal.h", "smol_device.h", "smol_rows.h", "smol_rows_rgb.h", "smol_rows_yuv.h",
           "smol_magic.h", "smol_tokens_device.h", "smol_patch.h", "smol_patch_kernels.h"]

# -ffp-contract=off: the kernels round every multiply and add on their own, as
# the definition does; fused multiply-adds are never formed implicitly.
# Packed fp32 VALU ops are disabled for the device code (the compiler would
# otherwise form v_pk_fma/mul/add_f32 from ordinary float code). The host pass
# warns that it does not know the feature; that warning is harmless.
HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-Wall",
    "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]
# Per-file additions. The fp16 contiguous-walk RGB kernels (c2, c3 and the
# low-resolution op's second launch) are scheduled for instruction-level
# parallelism instead of occupancy: same registers' occupancy, c3 81.2 ->
# 79.2 us per step (three alternations on one box), the others unchanged;
# the fp32 kernels lost 1 % with it, so they keep the default.
FILE_FLAGS = {
    "smol_rows_rgb_f16_range.hip": ["-mllvm", "-amdgpu-sched-strategy=max-ilp"],
}
LINK_FLAGS = ["--offload-arch=gfx950", "-shared", "-fPIC"]


def hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found; ROCm is required to build libsmol")


def _jobs() -> int:
    try:
        n = int(os.environ.get("MAX_JOBS", ""))
    except ValueError:
        n = 0
    return max(1, min(n or (os.cpu_count() or 4), 16))


def _noise_free(stderr: str) -> str:
    noise = ("is not a recognized feature for this target", "kernel-resource-usage")
    return "\n".join(line for line in stderr.splitlines() if not any(n in line for n in noise))


# Device code is compiled with the compiler's per-kernel resource remarks; a
# kernel that spills to or keeps a struct in private memory (scratch) fails the
# build: every access would be a memory round trip on the hot path.
RESOURCE_REMARKS = "-Rpass-analysis=kernel-resource-usage"


def _scratch_users(stderr: str) -> list:
    users, name = [], None
    for line in stderr.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            name = m.group(1)
            continue
        m = re.search(r"ScratchSize \[bytes/lane\]: (\d+)", line)
        if m and int(m.group(1)) > 0:
            users.append(f"{name}: {m.group(1)} bytes/lane")
    return users


def build_pycall(verbose: bool = False) -> str:
    """The CPython extension of the binding (host code only)."""
    cc = shutil.which("gcc") or shutil.which("cc") or hipcc()
    tmp = PYCALL + ".tmp"
    cmd = [cc, "-O2", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-o",
           tmp, os.path.join(CSRC, "smol_pycall.c")]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"building _smolcall failed ({res.returncode}):\n{res.stderr}")
    os.replace(tmp, PYCALL)
    return PYCALL


def rocm_torch() -> str | None:
    """The folder of the installed torch, None without one for ROCm."""
    try:
        import torch
    except ImportError:
        return None
    return os.path.dirname(torch.__file__) if torch.version.hip else None


def pytokens_command() -> list | None:
    """The compiler call of the token operators' binding (host code only,
    against the headers and libraries of the installed torch); None where there
    is no torch to bind: the C library needs none."""
    base = rocm_torch()
    if base is None:
        return None
    import torch
    libs = os.path.join(base, "lib")
    cc = shutil.which("g++") or hipcc()
    return [cc, "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__",
            "-DUSE_ROCM", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-I", sysconfig.get_paths()["include"], "-I", INCLUDE,
            "-isystem", os.path.join(base, "include"),
            "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
            "-isystem", os.path.join(os.path.dirname(os.path.dirname(hipcc())), "include"),
            os.path.join(CSRC, "smol_tokens_py.cpp"), "-L", libs, "-Wl,--no-as-needed",
            "-ltorch_python", "-ltorch_cpu", "-ltorch_hip", "-lc10_hip", "-lc10"]


def build(verbose: bool = False) -> str:
    cc = hipcc()
    build_pycall(verbose)
    pytokens = pytokens_command()
    if pytokens is None:
        print("no torch for ROCm: the token operators' Python binding is not built",
              file=sys.stderr, flush=True)
        return _build_library(cc, verbose)
    # beside the kernels: torch's headers take a while
    pytokens += ["-o", PYTOKENS + ".tmp"]
    if verbose:
        print(" ".join(pytokens), flush=True)
    binding = subprocess.Popen(pytokens, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    try:
        return _build_library(cc, verbose)
    finally:
        _, err = binding.communicate()
        if binding.returncode != 0:
            raise RuntimeError(f"building _smoltokens failed ({binding.returncode}):\n{err}")
        os.replace(PYTOKENS + ".tmp", PYTOKENS)


def _build_library(cc: str, verbose: bool) -> str:
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory(prefix="smol_build_") as objdir:
        cmds = []
        for src in SOURCES:
            obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
            remarks = [RESOURCE_REMARKS] if src.endswith(".hip") else []
            cmds.append((obj, [cc, *HIPCC_FLAGS, *FILE_FLAGS.get(src, []), *remarks, "-I", INCLUDE,
                               "-I", CSRC, "-c", "-o", obj, os.path.join(CSRC, src)]))
        pending = list(cmds)
        running = []
        errors = []
        while pending or running:
            while pending and len(running) < _jobs():
                obj, cmd = pending.pop(0)
                if verbose:
                    print(" ".join(cmd), flush=True)
                running.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE,
                                                      stderr=subprocess.PIPE, text=True)))
            cmd, proc = running.pop(0)
            _, err = proc.communicate()
            scratch = _scratch_users(err)
            err = _noise_free(err)
            if proc.returncode != 0:
                errors.append(f"{cmd[-1]} ({proc.returncode}):\n{err}")
            elif scratch:
                errors.append(f"{cmd[-1]}: kernels using scratch memory:\n" + "\n".join(scratch))
            elif verbose and err.strip():
                print(err, file=sys.stderr)
        if errors:
            raise RuntimeError("hipcc failed:\n" + "\n".join(errors))
        link = [cc, *LINK_FLAGS, "-o", tmp, *[obj for obj, _ in cmds]]
        if verbose:
            print(" ".join(link), flush=True)
        res = subprocess.run(link, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"link failed ({res.returncode}):\n{_noise_free(res.stderr)}")
    os.replace(tmp, LIB)
    return LIB


def sources_newer_than_lib() -> bool:
    built = [LIB, PYCALL] + ([PYTOKENS] if rocm_torch() else [])
    if not all(os.path.exists(f) for f in built):
        return True
    t = min(os.path.getmtime(f) for f in built)
    files = [os.path.join(CSRC, f)
             for f in SOURCES + HEADERS + ["smol_pycall.c", "smol_tokens_py.cpp"]] + [
        os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE) if f.endswith(".h")]
    return any(os.path.getmtime(f) > t for f in files)


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
