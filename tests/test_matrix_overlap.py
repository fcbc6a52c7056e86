"""Buffers of the matrix operators that share elements are refused before anything is launched (no GPU; the addresses are never read)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2105_00619_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(B.LIB_PATH):
        from paper_2105_00619_amd import build
        build.build(verbose=False)


def test_shared_bytes_of_matrices_are_found(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path / "overlap_check")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
                        "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2105_00619_amd", "csrc"),
                        os.path.join(ROOT, "tests", "overlap_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout + r.stderr


ROWS, IN, OUT = 160, 64, 32
SIZES = {"x": (ROWS, IN), "w": (OUT, IN), "residual": (ROWS, OUT), "y": (ROWS, OUT), "z": (ROWS, OUT), "dy": (ROWS, OUT),
         "dx": (ROWS, IN), "dw": (OUT, IN), "bias": (1, OUT), "dbias": (1, OUT)}


def _apart():
    """fp32 arguments of both directions, every buffer at a place of its own."""
    a = B.optorch_linear_t()
    a.precision, a.activation, a.rows, a.in_features, a.out_features = 0, 2, ROWS, IN, OUT
    for i, (n, (_, cols)) in enumerate(SIZES.items()):
        setattr(a, n, (1 + i) << 30)
        if "bias" not in n:
            setattr(a, "ldr" if n == "residual" else "ld" + n, cols)
    a.workspace, a.workspace_bytes = 20 << 30, 1 << 30
    return a


@pytest.mark.parametrize("backward,written,other", [
    (0, "y", "x"), (0, "y", "w"), (0, "y", "z"), (0, "z", "x"), (0, "z", "w"), (0, "z", "residual"), (0, "y", "bias"), (0, "z", "bias"),
    (0, "y", "workspace"), (0, "x", "workspace"),
    (1, "dx", "dy"), (1, "dx", "x"), (1, "dx", "w"), (1, "dx", "z"), (1, "dx", "dw"), (1, "dw", "x"), (1, "dw", "w"), (1, "dw", "dy"),
    (1, "dw", "z"), (1, "dbias", "dx"), (1, "dbias", "dw"), (1, "dbias", "dy"), (1, "dw", "workspace"), (1, "w", "workspace"),
])
def test_linear_buffers_that_overlap(backward, written, other):
    lib = B.load_library()
    fn = lib.optorch_linear_backward if backward else lib.optorch_linear_forward
    for shift in (0, 4, -4):  # (from the last element of one to the first of the other, and whole)
        a = _apart()
        if other == "workspace":
            a.workspace = getattr(a, written)
        else:
            setattr(a, written, getattr(a, other) + shift)
        assert fn(C.byref(a)) == B.E_INVALID
        message = lib.optorch_matrix_last_error().decode()
        assert "overlap" in message and written in message and other in message
    # a skip connection that is not y as a whole
    a = _apart()
    a.residual = a.y + 4
    assert lib.optorch_linear_forward(C.byref(a)) == B.E_INVALID and "overlap" in lib.optorch_matrix_last_error().decode()


def test_flat_vectors_that_overlap():
    f = getattr(B.load_library(), "_ZN4oseq21ortho_vectors_overlapEPK13optorch_orthoPKviS4_i")
    f.argtypes, f.restype = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32], C.c_bool
    p = B.OrthoPlan([(10, 4, 6, 20), (100, 8, 8, 8)])
    at = 1 << 20
    assert f(p.handle, at, 0, at, 0) and f(p.handle, at, 0, at, 1) and f(p.handle, at, 1, at + 2, 1)
    assert f(p.handle, at, 0, at + 4 * (p.span - 11), 0)       # the last element of one matrix, the first of another
    assert not f(p.handle, at, 0, at + 4 * (p.span - 10), 0)
    assert not f(p.handle, at, 0, at + 4 * p.span, 0) and not f(p.handle, at + 4 * p.span, 1, at, 0)
    p.close()
    p = B.OrthoPlan([(0, 5, 6, 20)])
    assert not f(p.handle, at, 0, at + 4 * 6, 0) and f(p.handle, at, 0, at + 4 * 5, 0)  # side by side in shared rows
    p.close()
