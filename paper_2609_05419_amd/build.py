"""Build the HIP library libo2m.so in-tree for gfx950 (hipcc)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libo2m.so")
SOURCES = ["api.hip", "k_scale.hip", "k_residue.hip", "k_gemm.hip", "k_crt.hip", "moduli.cpp",
           "api_model.hip", "k_quant.hip", "k_fp8.hip", "k_fp8_scaled.hip", "k_fp8_partial.hip", "k_fp8_wide.hip",
           "k_fp8_few.hip", "k_ortho.hip", "k_ortho_small.hip"]
# measurement probes (the practical int8 MFMA ceiling, HBM streaming rates), a
# library of their own
PROBE_LIB = os.path.join(HERE, "libo2m_probe.so")
PROBE_SOURCES = ["probe_mfma.hip", "probe_hbm.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 instructions stay off: the compiler must not emit them
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def build(verbose: bool = False) -> str:
    _build_one(PROBE_LIB, PROBE_SOURCES, verbose)
    return _build_one(LIB, SOURCES, verbose)


def _run(cmd, verbose: bool, what: str) -> None:
    if verbose:
        print(" ".join(cmd))
    r = subprocess.run(cmd, capture_output=True, text=True)
    lines = [l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l]
    if r.returncode != 0:
        sys.stderr.write("\n".join(lines) + "\n")
        raise RuntimeError(f"hipcc failed building {what}")
    if verbose and lines:
        print("\n".join(lines))


def _build_one(lib: str, sources, verbose: bool) -> str:
    """One object per source, compiled side by side, then the library."""
    tmp = lib + ".tmp"
    with tempfile.TemporaryDirectory() as objs:
        def compile_one(src):
            obj = os.path.join(objs, src + ".o")
            _run([HIPCC, *FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", "-o", obj,
                  os.path.join(CSRC, src)], verbose, src)
            return obj
        with ThreadPoolExecutor(max_workers=min(len(sources), 8)) as pool:
            built = list(pool.map(compile_one, sources))
        _run([HIPCC, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp, *built], verbose, os.path.basename(lib))
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(verbose=True))
