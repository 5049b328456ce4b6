"""Builds libosdp.so (HIP, gfx950) with hipcc and the binding's _pointers.so (C) with gcc, in-tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libosdp.so"
POINTERS = PKG / "_pointers.so"
SOURCES = ["osdp_api.hip", "osdp_gather.hip", "osdp_gemm.hip", "osdp_epilogue.hip", "osdp_search.hip", "osdp_adamw.hip", "osdp_int8.hip", "osdp_qk.hip"]
HEADERS = [CSRC / "osdp_internal.h", CSRC / "activation.h", CSRC / "gemm_launch.h", CSRC / "gemm_common.h", CSRC / "gemm_dma.h", CSRC / "gemm_i8.h", CSRC / "gemm_i8_w4.h", CSRC / "gemm_skinny.h", CSRC / "gemm_w4.h", CSRC / "gemm_w4p.h", ROOT / "include" / "osdp.h"]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-fvisibility=hidden",
    "-Wall", "-Wno-unused-function",
    # keep the compiler from forming packed-fp32 VALU ops
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not Path(exe).exists():
        raise RuntimeError("hipcc not found: libosdp cannot be built")
    return exe


def is_stale() -> bool:
    if not LIB.exists():
        return True
    t = LIB.stat().st_mtime
    deps = [CSRC / s for s in SOURCES] + HEADERS
    return any(d.stat().st_mtime > t for d in deps)


def build_pointers() -> Path:
    """Compile csrc/pointers.c into paper_2209_13258_amd/_pointers.so, a module of the Python that runs."""
    tmp = POINTERS.with_suffix(f".so.tmp{os.getpid()}")
    subprocess.run(["gcc", "-O2", "-std=c11", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall", "-Wextra", "-Wno-missing-field-initializers",
                    f"-I{sysconfig.get_paths()['include']}", f"-I{ROOT / 'include'}", str(CSRC / "pointers.c"), "-o", str(tmp)], check=True)
    os.replace(tmp, POINTERS)
    return POINTERS


def build(force: bool = True, verbose: bool = False) -> Path:
    """Compile every HIP source into paper_2209_13258_amd/libosdp.so, and the binding's module."""
    if force or not POINTERS.exists() or POINTERS.stat().st_mtime < (CSRC / "pointers.c").stat().st_mtime:
        build_pointers()
    if not force and not is_stale():
        return LIB
    tmp = LIB.with_suffix(f".so.tmp{os.getpid()}")
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        made = [str(Path(objects) / Path(s).with_suffix(".o")) for s in SOURCES]
        list(pool.map(lambda s, o: _hipcc(["-c", str(CSRC / s), "-o", o], verbose), SOURCES, made))
        _hipcc(["-shared", *made, "-o", str(tmp)], verbose)
    os.replace(tmp, LIB)
    return LIB


def _hipcc(args, verbose: bool) -> None:
    cmd = [hipcc(), *HIPCC_FLAGS, f"-I{ROOT / 'include'}", f"-I{CSRC}", *args]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed:\n{err}")
    if verbose and err.strip():
        print(err)


if __name__ == "__main__":
    print(build(force=True, verbose=True))
