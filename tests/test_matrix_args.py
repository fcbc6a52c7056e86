"""Host-side checks of the matrix operators (no GPU): plans, workspace sizes and refusals.  A refused call launches nothing, so
the pointers need not be device memory."""
import ctypes as C
import os

import pytest

from paper_2105_00619_amd import binding as B
from paper_2105_00619_amd.binding import E_BUDGET, E_INVALID, E_ORDER, OK, OptorchError, OrthoPlan


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(B.LIB_PATH):
        from paper_2105_00619_amd import build
        build.build(verbose=False)


def _linear(**kw):
    """Arguments of both directions that pass every check; the addresses are never read."""
    a = B.optorch_linear_t()
    a.precision, a.activation, a.rows, a.in_features, a.out_features = 1, 2, 160, 64, 32
    for n, cols in (("x", 64), ("w", 64), ("residual", 32), ("y", 32), ("z", 32), ("dy", 32), ("dx", 64), ("dw", 64)):
        setattr(a, n, 1 << 20)
        setattr(a, "ldr" if n == "residual" else "ld" + n, cols)
    a.bias = a.dbias = 1 << 20
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_workspace_of_aligned_16_bit_operands_holds_no_copies():
    lib = B.load_library()
    assert lib.optorch_linear_workspace(C.byref(_linear(rows=65536, in_features=512, out_features=512, ldx=512, ldw=512, ldy=512,
                                                        ldz=512, ldr=512)), 0) == 0
    # rows that are no multiple of 16 bytes apart, and addresses off a 16-byte boundary, are laid out anew
    odd = lib.optorch_linear_workspace(C.byref(_linear(ldx=65)), 0)
    assert odd >= 160 * 64 * 2
    assert lib.optorch_linear_workspace(C.byref(_linear(x=(1 << 20) + 2)), 0) == odd
    # fp32: three planes of each operand
    assert lib.optorch_linear_workspace(C.byref(_linear(precision=0)), 0) >= (160 + 32) * 64 * 6
    # backward with an activation keeps dz
    assert lib.optorch_linear_workspace(C.byref(_linear()), 1) >= 160 * 32 * 2
    # a forward pass of few samples reads its operands as they lie
    assert lib.optorch_linear_workspace(C.byref(_linear(rows=16, ldx=65, precision=0)), 0) == 0
    assert lib.optorch_linear_workspace(C.byref(_linear(rows=0)), 0) == 0


@pytest.mark.parametrize("kw,backward,word", [
    (dict(precision=3), 0, "precision"), (dict(precision=-1), 1, "precision"),
    (dict(activation=4), 0, "activation"), (dict(activation=-1), 1, "activation"),
    (dict(rows=-1), 0, "rows"), (dict(rows=1 << 31), 0, "rows"),
    (dict(in_features=0), 0, "features"), (dict(out_features=0), 1, "features"), (dict(in_features=1 << 22), 0, "features"),
    (dict(x=None), 0, "x"), (dict(w=None), 0, "w"), (dict(y=None), 0, "y"),
    (dict(ldx=63), 0, "leading dimension of x"), (dict(ldw=63), 0, "leading dimension of w"), (dict(ldy=31), 0, "leading dimension of y"),
    (dict(ldz=31), 0, "leading dimension of z"), (dict(ldr=31), 0, "leading dimension of residual"),
    (dict(ldx=1 << 22), 0, "leading dimension of x"),
    (dict(x=(1 << 20) + 1), 0, "aligned"), (dict(bias=(1 << 20) + 2), 0, "aligned"), (dict(precision=0, y=(1 << 20) + 2), 0, "aligned"),
    (dict(dy=None), 1, "dy"), (dict(z=None), 1, "z"), (dict(x=None), 1, "x"), (dict(w=None), 1, "w"),
    (dict(lddy=31), 1, "leading dimension of dy"), (dict(lddx=63), 1, "leading dimension of dx"),
    (dict(lddw=63), 1, "leading dimension of dw"), (dict(dbias=(1 << 20) + 1), 1, "aligned"),
    (dict(dx=None, dw=None, dbias=None), 1, "no gradient"),
])
def test_linear_refusals(kw, backward, word):
    lib = B.load_library()
    a = _linear(**kw)
    assert lib.optorch_linear_workspace(C.byref(a), backward) == E_INVALID
    assert word in lib.optorch_matrix_last_error().decode()
    fn = lib.optorch_linear_backward if backward else lib.optorch_linear_forward
    assert fn(C.byref(a)) == E_INVALID
    assert word in lib.optorch_matrix_last_error().decode()


def test_fp32_rows_of_planes_stay_inside_32_bit_offsets():
    """256 rows of a tile are addressed by 32-bit offsets, and a row of fp32 values as planes takes 8 bytes a value."""
    lib = B.load_library()
    most = (1 << 20) - 16
    assert 256 * 8 * most < 1 << 31 < 256 * 8 * (most + 16) + 1
    wide = dict(ldx=most + 1, ldw=most + 1, lddx=most + 1, lddw=most + 1)
    long = dict(ldy=most + 1, ldz=most + 1, ldr=most + 1, lddy=most + 1)
    for backward in (0, 1):
        for name, lds in (("in_features", wide), ("out_features", long)):
            assert lib.optorch_linear_workspace(C.byref(_linear(precision=0, **{name: most}, **lds)), backward) > 0
            assert lib.optorch_linear_workspace(C.byref(_linear(precision=0, **{name: most + 1}, **lds)), backward) == E_INVALID
            assert "fp32" in lib.optorch_matrix_last_error().decode()
            assert lib.optorch_linear_workspace(C.byref(_linear(**{name: most + 1}, **lds)), backward) >= 0


def test_linear_refuses_a_missing_small_or_misaligned_workspace():
    lib = B.load_library()
    a = _linear(precision=0)
    n = lib.optorch_linear_workspace(C.byref(a), 0)
    assert n > 0
    for p, size, code in ((None, n, E_INVALID), (1 << 20, n - 1, E_BUDGET), ((1 << 20) + 128, n, E_INVALID)):
        a.workspace, a.workspace_bytes = p, size
        assert lib.optorch_linear_forward(C.byref(a)) == code
        assert "workspace" in lib.optorch_matrix_last_error().decode()
    assert lib.optorch_linear_forward(None) == E_INVALID
    assert lib.optorch_linear_workspace(None, 0) == E_INVALID


def test_unused_operands_may_be_absent():
    lib = B.load_library()
    # without an activation the slope needs no z; without dw no x; without dx no w
    a = _linear(activation=0, z=None, x=None, dw=None)
    assert lib.optorch_linear_workspace(C.byref(a), 1) >= 0
    a = _linear(dx=None, w=None)
    assert lib.optorch_linear_workspace(C.byref(a), 1) >= 0
    a = _linear(z=None, residual=None, bias=None)
    assert lib.optorch_linear_workspace(C.byref(a), 0) >= 0


def test_ortho_plan_spans_and_packs():
    p = OrthoPlan([(64, 27), (8, 72), (10, 8)])
    assert p.span == 64 * 27 + 8 * 72 + 10 * 8
    assert p.workspace_bytes > 0
    p.close()
    # a matrix at an offset, rows further apart than they are long
    p = OrthoPlan([(100, 4, 6, 10)])
    assert p.span == 100 + 3 * 10 + 6
    p.close()
    # a wide matrix costs two iterates of two fp16 planes, no more than a few m x m matrices beside them
    p = OrthoPlan([(64, 65536)])
    assert 2 * 4 * 64 * 65536 <= p.workspace_bytes < 3 * 4 * 64 * 65536
    p.close()
    p = OrthoPlan([(64, 65536)], steps=3)
    assert p.workspace_bytes < 2 * 4 * 64 * 65536
    p.close()


@pytest.mark.parametrize("mats,kw,word", [
    ([], {}, "empty"),
    ([(0, 4)], {}, "rows and cols"), ([(4, 0)], {}, "rows and cols"), ([((1 << 20) + 1, 4)], {}, "rows and cols"),
    ([(40000, 40000)], {}, "shorter side"),
    ([(-1, 4, 4, 4)], {}, "offset"), ([(0, 4, 4, 3)], {}, "leading dimension"),
    ([(0, 4, 4, 4), (15, 4, 4, 4)], {}, "overlap"), ([(15, 4, 4, 4), (0, 4, 4, 4)], {}, "overlap"),
    ([(0, 4, 4, 10), (3, 4, 4, 10)], {}, "overlap"), ([(0, 4, 4, 10), (7, 4, 4, 10)], {}, "overlap"),
    ([(0, 4, 4, 10), (4, 4, 4, 9)], {}, "overlap"),
    ([(4, 4)], dict(steps=17), "steps"),
    ([(4, 4)], dict(coefficients=(float("nan"), 0, 0)), "finite"),
    ([(4, 4)], dict(eps=float("inf")), "eps"),
    ([(4, 4)], dict(coefficients=(20.0, 1.0, 1.0)), "singular value"),
])
def test_ortho_refusals(mats, kw, word):
    with pytest.raises(OptorchError) as e:
        OrthoPlan(mats, **kw)
    assert e.value.code == E_INVALID and word in str(e.value)


def test_ortho_accepts_matrices_side_by_side():
    OrthoPlan([(0, 4, 4, 10), (4, 4, 6, 10)]).close()
    OrthoPlan([(0, 4, 4, 4), (16, 4, 4, 4)]).close()
    OrthoPlan([(0, 2, 4, 10), (20, 2, 10, 10)]).close()


def test_ortho_call_order_and_arguments():
    lib = B.load_library()
    p = OrthoPlan([(4, 4)])
    m = B.optorch_muon_t()
    m.g = m.w = m.v = 1 << 20
    m.lr = 0.1
    assert lib.optorch_orthogonalize(p.handle, 0, 1 << 20, 0, 1 << 20, None) == E_ORDER
    assert lib.optorch_muon_update(p.handle, C.byref(m), None) == E_ORDER
    assert lib.optorch_ortho_bind(p.handle, None, 1 << 30) == E_INVALID
    assert lib.optorch_ortho_bind(p.handle, (1 << 20) + 64, 1 << 30) == E_INVALID
    assert lib.optorch_ortho_bind(p.handle, 1 << 20, p.workspace_bytes - 1) == E_BUDGET
    assert lib.optorch_ortho_bind(None, 1 << 20, 1 << 30) == E_INVALID
    assert lib.optorch_ortho_query(None, None, None) == E_INVALID
    assert lib.optorch_ortho_query(p.handle, None, None) == OK
    assert lib.optorch_orthogonalize(None, 0, 1 << 20, 0, 1 << 20, None) == E_INVALID
    assert lib.optorch_muon_update(None, C.byref(m), None) == E_INVALID
    p.close()
    lib.optorch_ortho_destroy(None)


def test_python_checks_name_what_is_wrong():
    import torch
    x, w = torch.zeros(3, 4), torch.zeros(5, 4)
    with pytest.raises(ValueError, match="GPU"):
        B.linear_forward(x, w)
    with pytest.raises(ValueError, match="activation"):
        B.linear_forward(x, w, activation="tanh")
    with pytest.raises(ValueError, match="need"):
        B.linear_backward(x, x, w, need=("dy",))
    with pytest.raises(ValueError, match="coefficients"):
        OrthoPlan([(4, 4)], steps=2, coefficients=[(1, 1, 1)])
