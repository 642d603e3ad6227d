"""Build libmita.so (the HIP/gfx950 MiTA library) in-tree with hipcc.

    python -m paper_2602_01219_amd.build [--jobs N]

Objects are compiled in parallel into paper_2602_01219_amd/_build/ and linked
into paper_2602_01219_amd/libmita.so. Always recompiles.
"""
from __future__ import annotations

import argparse
import os
import re
import shutil
import struct
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libmita.so")
ARCH = "gfx950"

SOURCES = ["mita_api.hip", "pool_scores.hip", "topk.hip", "select.hip", "route_attend.hip", "backward.hip", "tome.hip",
           "dense_forward.hip", "dense_backward.hip", "dense_prefix.hip", "norm.hip", "rms.hip",
           "rope.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
OBJDUMP = os.environ.get("LLVM_OBJDUMP", "/opt/rocm/llvm/bin/llvm-objdump")
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-fPIC", "-std=c++17",
    # no packed fp32 arithmetic in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
    "-Wno-unused-command-line-argument",
]
# MFMA accumulators in ordinary VGPRs: no copies between AGPRs and VGPRs around
# the VALU work on the same values. Not for the dense attention: kernels of two
# waves per SIMD get that form anyway, and the fp32 ones of one wave are slower with
# it (forward of 16 heads of 2048 tokens, d = 128: 290 us against 270).
VGPR_FORM = ["-Xarch_device", "-mllvm=-amdgpu-mfma-vgpr-form=1"]

# Matrix instructions that kernels may use: at most 32 cycles long. An instruction
# whose third operand is not its result's registers reads it while it runs, and
# nothing holds back an LDS read behind it that writes those registers: the compiler
# sets no wait for it. Of these three such a read came too late to be seen, whatever
# was in flight before them (operands in VGPRs and AGPRs, after chains of 0 to 64, one
# and two waves on each SIMD of the card); the 64 cycles of v_mfma_f32_32x32x2_f32 took
# the read's value every time. With the forced
# form an fp32 dQ kernel of that instruction (d = 128) had its row sums' last copies
# overwritten so: dQ off by 12% on four of 32 keys.
MFMA = {"v_mfma_f32_16x16x4_f32", "v_mfma_f32_16x16x32_bf16", "v_mfma_f32_32x32x16_bf16"}


def flags_for(src):
    return FLAGS if src.startswith("dense_") else FLAGS + VGPR_FORM


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = (r.stdout + r.stderr).strip()
    # the host pass does not know the device-only target feature; that note is harmless
    lines = [l for l in out.splitlines() if "packed-fp32-ops" not in l]
    return r.returncode, "\n".join(lines)


def code_objects(path):
    """The gfx950 code objects in a host object or library."""
    with open(path, "rb") as f:
        data = f.read()
    magic, at = b"__CLANG_OFFLOAD_BUNDLE__", 0
    while (at := data.find(magic, at)) >= 0:
        n, p = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            target = data[p + 24:p + 24 + length].decode()
            p += 24 + length
            if size and target.endswith(ARCH):
                yield data[at + offset:at + offset + size]
        at += len(magic)


def matrix_instructions(path):
    """Names of the matrix instructions in a host object or library."""
    names = set()
    for code in code_objects(path):
        with tempfile.NamedTemporaryFile(suffix=".co") as f:
            f.write(code)
            f.flush()
            r = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", f.name], capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"llvm-objdump failed on {path}:\n{r.stderr}")
        names.update(re.findall(r"\bv_s?mfmac?_\w+", r.stdout))
    return names


def check_matrix_instructions(path):
    names = matrix_instructions(path)
    if not names:
        raise RuntimeError(f"no {ARCH} matrix instructions found in {path}")
    other = names - MFMA
    if other:
        raise RuntimeError(f"{path} holds matrix instructions whose operands were not checked (MFMA): {sorted(other)}")


def build(jobs: int | None = None, verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    objs = []

    def compile_one(src):
        obj = os.path.join(BUILD, src.replace(".hip", ".o"))
        cmd = [HIPCC, *flags_for(src), "-c", os.path.join(CSRC, src), "-o", obj]
        rc, out = _run(cmd)
        if rc != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{out}")
        if verbose and out:
            print(out)
        return obj

    with ThreadPoolExecutor(max_workers=jobs or min(8, len(SOURCES))) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp"
    rc, out = _run([HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs])
    if rc != 0:
        raise RuntimeError(f"link failed:\n{out}")
    check_matrix_instructions(tmp)
    os.replace(tmp, LIB)
    return LIB


def clean():
    shutil.rmtree(BUILD, ignore_errors=True)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--jobs", type=int, default=None)
    ap.add_argument("-v", "--verbose", action="store_true")
    a = ap.parse_args()
    print(build(a.jobs, a.verbose))
    sys.exit(0)
