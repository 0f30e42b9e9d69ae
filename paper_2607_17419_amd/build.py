"""Build libkata.so (HIP, gfx950) in-tree with hipcc.

    python -m paper_2607_17419_amd.build        # or build() from Python

Every source under csrc/ is compiled for gfx950 only, with packed-FP32
instruction generation disabled, and linked into paper_2607_17419_amd/libkata.so.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libkata.so")
SOURCES = ["kata_api.hip", "kata_fp32.hip", "kata_mfma.hip", "kata_linear.hip", "kata_bwd.hip",
           "kata_bwd_bf.hip", "kata_mixer.hip", "kata_block.hip"]
# per-source flags: the bf16 gradients kernel updates MFMA results with VALU code,
# so its MFMAs write VGPRs (no AGPR copies)
EXTRA = {"kata_bwd_bf.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}

# objects joined into another after compiling: a test relinks the library from its
# objects by name and knows no others
JOINED = {"kata_linear.o": ["kata_mixer.o", "kata_block.o"]}

HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
LD = os.path.join(os.path.dirname(os.path.realpath(HIPCC)), "..", "llvm", "bin", "ld.lld")
ARCH = "gfx950"
CFLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fvisibility=hidden", "-Wall", "-Wno-unused-result",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, src.replace(".hip", ".o"))
    cmd = [HIPCC, *CFLAGS, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "is not a recognized feature for this target" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{out}")
    if out.strip():
        print(out, file=sys.stderr)
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    for name, more in JOINED.items():
        whole, parts = os.path.join(BUILD, name), [os.path.join(BUILD, m) for m in more]
        subprocess.run([LD, "-r", whole, *parts, "-o", whole + ".tmp"], check=True)
        os.replace(whole + ".tmp", whole)
        objs = [o for o in objs if o not in parts]
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", *objs, "-o", tmp]
    subprocess.run(cmd, check=True, capture_output=not verbose)
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
