"""Host build of the 8-bit products' plan (fp8_plan.h): splits cover k once and their sums fit
the scratch memory that the call asks for, and the shapes that the GPU tests take for split
ones are."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

pytest.importorskip("torch")
import paper_2609_05419_amd as o2m  # noqa: E402
from fp8_shapes import SPLIT, SPLIT_LINEAR

HERE = os.path.dirname(os.path.abspath(__file__))
KINDS = [(0, 2), (0, 0), (1, 1), (1, 0)]   # scales, type of the result


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    out = tmp_path_factory.mktemp("plan") / "libfp8_plan_host.so"
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-I", os.path.join(HERE, "..", "include"),
                    os.path.join(HERE, "fp8_plan_host.cpp"), "-o", str(out)], check=True)
    lib = ctypes.CDLL(str(out))

    def call(m, n, k, kind):
        v = np.zeros(5, dtype=np.int32)
        lib.t_plan_fp8(m, n, k, kind[0], kind[1], ctypes.c_void_p(v.ctypes.data))
        return dict(zip(("few", "rows", "cols", "splits", "per"), (int(x) for x in v)))
    return call


@pytest.mark.parametrize("kind", KINDS)
def test_splits_cover_k(plan, kind):
    rng = np.random.default_rng(1)
    for _ in range(400):
        m, n, k = (int(v) for v in np.exp(rng.uniform(0, [9.1, 9.1, 12.0])).astype(np.int64))
        p = plan(m, n, k, kind)
        blocks = -(-k // 128)
        assert p["few"] == (min(m, n) <= 32)
        assert (p["splits"] - 1) * p["per"] < blocks <= p["splits"] * p["per"]
        if p["splits"] > 1:
            assert not p["few"] and (p["rows"], p["cols"]) == (64, 64) and p["splits"] <= 16
            # what the call asks for holds the sums of either order
            assert o2m._L.o2m_gemm_fp8_workspace(m, n, k) >= 4 * p["splits"] * m * (-(-n // 4) * 4)
            assert o2m._L.o2m_gemm_fp8_workspace(n, m, k) >= 4 * p["splits"] * m * (-(-n // 4) * 4)


@pytest.mark.parametrize("m,n,k,splits", SPLIT)
def test_split_shapes(plan, m, n, k, splits):
    for kind, want in zip(KINDS, splits):   # either order of the result
        assert plan(m, n, k, kind)["splits"] == plan(n, m, k, kind)["splits"] == want


@pytest.mark.parametrize("tokens,n,k", SPLIT_LINEAR)
def test_split_layers(plan, tokens, n, k):
    for kind in KINDS:
        assert plan(tokens, n, k, kind)["splits"] > 1
