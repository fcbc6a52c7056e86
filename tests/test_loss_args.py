"""Host-side checks of the losses over many classes (no GPU): workspace sizes, pieces and refusals.  A refused call launches nothing, so
the pointers need not be device memory."""
import ctypes as C
import os

import pytest

from paper_2105_00619_amd import binding as B
from paper_2105_00619_amd.binding import E_BUDGET, E_INVALID

AT = {n: (1 + i) << 26 for i, n in enumerate(("x", "w", "dx", "dw", "teacher", "indices", "bias", "labels", "loss", "lse", "dloss", "dbias"))}
WS = 1 << 34


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(B.LIB_PATH):
        from paper_2105_00619_amd import build
        build.build(verbose=False)


def _loss(distill=False, **kw):
    """Arguments of both directions that pass every check; the addresses are never read."""
    a = B.optorch_softmax_loss_t()
    a.precision, a.teacher_precision, a.rows, a.in_features, a.classes = 1, 2, 160, 64, 500
    for n, v in AT.items():
        setattr(a, n, v)
    a.ldx = a.ldw = a.lddx = a.lddw = 64
    a.top, a.temperature, a.ldi, a.ldt = 8, 2.0, 8, 8
    if distill:
        a.labels = None
    else:
        a.indices = a.teacher = None
    a.workspace, a.workspace_bytes = WS, 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,backward,word", [
    (dict(precision=3), 0, "precision"), (dict(precision=-1), 1, "precision"), (dict(rows=-1), 0, "rows"), (dict(rows=1 << 31), 1, "rows"),
    (dict(in_features=0), 0, "in_features"), (dict(classes=0), 1, "classes"), (dict(classes=1 << 22), 0, "classes"),
    (dict(precision=0, classes=1 << 20), 0, "fp32"), (dict(precision=0, in_features=1 << 20), 1, "fp32"),
    (dict(x=None), 0, "null x"), (dict(w=None), 1, "null w"), (dict(lse=None), 0, "null lse"), (dict(lse=None), 1, "null lse"), (dict(loss=None), 0, "null loss"),
    (dict(dloss=None), 1, "null dloss"), (dict(labels=None), 0, "neither"), (dict(indices=AT["indices"]), 0, "exclude"), (dict(teacher=AT["teacher"]), 1, "exclude"),
    (dict(dx=None, dw=None, dbias=None), 1, "no gradient"),
    (dict(ldx=63), 0, "leading dimension of x"), (dict(ldw=63), 0, "leading dimension of w"), (dict(lddx=63), 1, "leading dimension of dx"),
    (dict(lddw=1 << 22), 1, "leading dimension of dw"), (dict(x=AT["x"] + 1), 0, "aligned"), (dict(precision=0, w=AT["w"] + 2), 0, "aligned"),
    (dict(bias=AT["bias"] + 2), 0, "aligned"), (dict(labels=AT["labels"] + 1), 0, "aligned"), (dict(dbias=AT["dbias"] + 1), 1, "aligned"),
    (dict(label_smoothing=-0.1), 0, "label_smoothing"), (dict(label_smoothing=1.1), 1, "label_smoothing"), (dict(label_smoothing=NAN), 0, "label_smoothing"),
    (dict(z_loss=-1.0), 0, "z_loss"), (dict(z_loss=INF), 1, "z_loss"), (dict(z_loss=NAN), 0, "z_loss"),
    (dict(workspace=None), 1, "null workspace"), (dict(workspace=WS + 128), 0, "256-byte"),
    (dict(loss=AT["lse"]), 0, "loss"), (dict(lse=AT["x"] + 64), 0, "x and lse"), (dict(loss=AT["labels"] + 4), 0, "labels and loss"),
    (dict(dx=AT["x"]), 1, "x and dx"), (dict(dw=AT["w"]), 1, "w and dw"), (dict(dw=AT["dx"] + 128), 1, "dx and dw"), (dict(dbias=AT["bias"]), 1, "bias and dbias"),
    (dict(dx=AT["dloss"]), 1, "dloss and dx"), (dict(workspace=AT["x"]), 1, "x and workspace"), (dict(workspace=AT["labels"]), 0, "labels and workspace"),
])
def test_refusals(kw, backward, word):
    lib = B.load_library()
    fn = lib.optorch_softmax_loss_backward if backward else lib.optorch_softmax_loss_forward
    assert fn(C.byref(_loss(**kw))) == E_INVALID
    assert word in lib.optorch_matrix_last_error().decode()


@pytest.mark.parametrize("kw,backward,word", [
    (dict(teacher_precision=3), 0, "teacher_precision"), (dict(top=0), 0, "top"), (dict(top=1025, ldi=1025, ldt=1025), 1, "top"),
    (dict(temperature=0.0), 0, "temperature"), (dict(temperature=-1.0), 1, "temperature"), (dict(temperature=NAN), 0, "temperature"),
    (dict(temperature=INF), 0, "temperature"), (dict(temperature=1e-40), 1, "temperature"),
    (dict(label_smoothing=0.1), 0, "go with labels"), (dict(z_loss=0.1), 1, "go with labels"),
    (dict(indices=None), 0, "null indices"), (dict(teacher=None), 1, "null teacher"), (dict(ldi=7), 0, "leading dimension of indices"),
    (dict(ldt=7), 1, "leading dimension of teacher"), (dict(indices=AT["indices"] + 2), 0, "aligned"), (dict(teacher=AT["teacher"] + 1), 0, "aligned"),
    (dict(loss=AT["teacher"] + 4), 0, "teacher and loss"), (dict(dx=AT["indices"]), 1, "indices and dx"),
])
def test_refusals_of_a_teacher(kw, backward, word):
    lib = B.load_library()
    fn = lib.optorch_softmax_loss_backward if backward else lib.optorch_softmax_loss_forward
    assert fn(C.byref(_loss(distill=True, **kw))) == E_INVALID
    assert word in lib.optorch_matrix_last_error().decode()


@pytest.mark.parametrize("teacher", [False, True])
@pytest.mark.parametrize("backward", [0, 1])
def test_null_arguments_and_a_short_workspace(teacher, backward):
    lib = B.load_library()
    fn = lib.optorch_softmax_loss_backward if backward else lib.optorch_softmax_loss_forward
    assert fn(None) == E_INVALID and lib.optorch_softmax_loss_workspace(None, backward) == E_INVALID
    n = lib.optorch_softmax_loss_workspace(C.byref(_loss(teacher)), backward)
    assert n > 0 and n % 256 == 0
    assert fn(C.byref(_loss(teacher, workspace_bytes=n - 1))) == E_BUDGET
    assert lib.optorch_softmax_loss_workspace(C.byref(_loss(teacher, rows=0)), backward) == 0


def _shape(a, backward):
    """Edge of a logits tile, pieces of the classes, tiles and parts of dx and dw (loss.cpp)."""
    fn = B.load_library()["_ZN4oseq10loss_shapeEPK22optorch_softmax_loss_tbPi"]
    fn.argtypes, fn.restype = [C.POINTER(B.optorch_softmax_loss_t), C.c_bool, C.c_int32 * 4], None
    out = (C.c_int32 * 4)()
    fn(C.byref(a), bool(backward), out)
    return list(out)


def test_the_workspace_does_not_grow_with_the_logits():
    """Forward a row's sums and its target's logits, backward half a GB of ds at a time, whatever the classes."""
    lib = B.load_library()
    size = lambda b, **kw: lib.optorch_softmax_loss_workspace(C.byref(_loss(rows=65536, in_features=512, ldx=512, ldw=512, lddx=512, lddw=512, **kw)), b)  # noqa: E731
    for classes in (32000, 128000, 1000000):
        logits = 65536 * classes * 4
        assert size(0, classes=classes) <= logits / 60
        assert size(1, classes=classes) <= (600 << 20) + 65536 * 512 * 8 + (1 << 26)
        assert _shape(_loss(rows=65536, classes=classes), True)[1] >= 65536 * classes * 2 / (512 << 20)
    assert _shape(_loss(), True)[1] == 1 and _shape(_loss(), False)[1] == 1


def test_sizes_take_the_tiles_that_the_gpu_tests_are_for():
    shape = lambda rows, cin, classes, p, b: _shape(_loss(precision=p, rows=rows, in_features=cin, classes=classes, ldx=cin, ldw=cin, lddx=cin, lddw=cin), b)  # noqa: E731
    for p in (0, 1, 2):
        assert [shape(*n, p, 1)[0] for n in ((520, 256, 2050), (300, 800, 50001), (2300, 712, 7001))] == [64, 128, 256]
        assert [shape(*n, p, 0)[0] for n in ((520, 256, 2050), (300, 800, 50001), (2300, 712, 7001))] == [64, 128, 256]
    assert shape(2300, 712, 7001, 0, 1)[3] // 1000 == 256
    assert shape(16400, 712, 17001, 1, 1) == [256, 2, 256001, 256005], "sums over two pieces, parts of a reduction"
    assert shape(16, 2048, 65536, 1, 0)[0] == 32, "the kernel that streams the weights counts in runs of 16"
    assert shape(16, 72, 700, 0, 0)[0] == 32, "few rows in fp32 too"


def test_gradients_asked_for_alone_are_cut_alike():
    for kw in (dict(), dict(rows=4096, in_features=2048, classes=100, ldx=2048, ldw=2048, lddx=2048, lddw=2048), dict(precision=0)):
        full = _shape(_loss(**kw), True)
        for off in (dict(dx=None), dict(dw=None), dict(dbias=None)):
            assert _shape(_loss(**kw, **off), True) == full
