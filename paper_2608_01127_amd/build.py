"""Build the HIP library libmw.so in-tree for gfx950.

    python -m paper_2608_01127_amd.build        (or build() from Python)

Every call recompiles.  Objects go to paper_2608_01127_amd/_build/, the
shared library to paper_2608_01127_amd/libmw.so.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libmw.so")

ARCH = "gfx950"
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", f"-I{os.path.join(ROOT, 'include')}",
          # packed fp32 VALU forms are kept out of the generated code
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Wno-unused-command-line-argument"]
# LLVM's iterative ILP scheduler measured faster for the D = 128 forward
# kernels (bf16 and e4m3) and slower for the D = 64 ones and for the D = 128
# backward grid (1% with its dK/dV work at two waves per SIMD); the attention
# sources are therefore compiled once per head dimension.
ILP = ["-mllvm", "-amdgpu-sched-strategy=iterative-ilp"]
UNITS = [  # (object name, source, extra flags)
    ("attn_fwd64", "attn_fwd.hip", ["-DMW_FWD_HEAD_DIM=64"]),
    ("attn_fwd72", "attn_fwd.hip", ["-DMW_FWD_HEAD_DIM=72"]),
    ("attn_fwd128", "attn_fwd.hip", ["-DMW_FWD_HEAD_DIM=128", *ILP]),
    # the 256-row cached configuration: 64-byte loop alignment measured faster
    ("attn_fwd128c", "attn_fwd.hip", ["-DMW_FWD_HEAD_DIM=128", "-DMW_FWD_CACHED", *ILP, "-falign-loops=64"]),
    # the tiles for grids that do not fill the card
    ("attn_fwd128s", "attn_fwd.hip", ["-DMW_FWD_HEAD_DIM=128", "-DMW_FWD_SMALL"]),
    ("attn_fwd128dec", "attn_fwd.hip", ["-DMW_FWD_HEAD_DIM=128", "-DMW_FWD_DECODE"]),
    ("attn_bwd64", "attn_bwd.hip", ["-DMW_BWD_HEAD_DIM=64"]),
    ("attn_bwd72", "attn_bwd.hip", ["-DMW_BWD_HEAD_DIM=72"]),
    ("attn_bwd128", "attn_bwd.hip", ["-DMW_BWD_HEAD_DIM=128"]),
    ("attn_fwd_fp8", "attn_fwd_fp8.hip", ILP),
    ("kvcache", "kvcache.hip", []),
    *((f"cross{d}", "attn_rows.hip", [f"-DMW_ROWS_HEAD_DIM={d}"]) for d in (64, 72, 128)),
    *((f"paged{d}", "attn_rows.hip", [f"-DMW_ROWS_HEAD_DIM={d}", "-DMW_ROWS_PAGED"]) for d in (64, 72, 128)),
    *((f"cross_bwd{d}", "attn_cross_bwd.hip", [f"-DMW_CROSS_HEAD_DIM={d}"]) for d in (64, 72, 128)),
    *((f"packed{d}", "attn_packed.hip", [f"-DMW_PACKED_HEAD_DIM={d}"]) for d in (64, 72, 128)),
    *((f"packed_bwd{d}", "attn_packed_bwd.hip", [f"-DMW_PACKED_HEAD_DIM={d}", "-DMW_SCALAR_LDS"]) for d in (64, 72, 128)),
    ("packed_plan", "packed_plan.hip", []),
    ("rope", "rope.hip", []),
    ("weigh", "weigh.hip", []),
    ("keep", "keep.hip", []),
    ("kvpages", "kvpages.hip", []),
    ("mw_cross", "mw_cross.cpp", []),
    ("mw_pages", "mw_pages.cpp", []),
    ("mw_packed", "mw_packed.cpp", []),
    ("mw_rope", "mw_rope.cpp", []),
    ("mw_api", "mw_api.cpp", []),
    ("sched", "sched.cpp", []),
]
SOURCES = sorted({u[1] for u in UNITS})


def _compile(unit, extra) -> str:
    name, src, flags = unit
    obj = os.path.join(BUILD, name + ".o")
    lang = ["-x", "hip"]
    cmd = [HIPCC, *lang, *COMMON, *flags, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False, extra=()) -> str:
    if not os.path.exists(HIPCC):
        raise RuntimeError(f"hipcc not found at {HIPCC}")
    os.makedirs(BUILD, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(UNITS))) as ex:
        objs = list(ex.map(lambda u: _compile(u, list(extra)), UNITS))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


def clean() -> None:
    shutil.rmtree(BUILD, ignore_errors=True)
    if os.path.exists(LIB):
        os.remove(LIB)


if __name__ == "__main__":
    build(verbose=True, extra=sys.argv[1:])
