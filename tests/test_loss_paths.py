"""Which of the forward pass' kernels a loss of few rows takes (no GPU): the sizes that the GPU tests name a kernel by."""
import ctypes as C

import pytest

from paper_2105_00619_amd import binding as B
from tests.test_loss_args import AT, _built, _loss  # noqa: F401


def _path(rows, cin, classes, precision=1, **kw):
    """0: tiles; 1: weights straight from memory; otherwise the blocks that stream them."""
    fn = B.load_library()["_ZN4oseq9loss_pathEPK22optorch_softmax_loss_t"]
    fn.argtypes, fn.restype = [C.POINTER(B.optorch_softmax_loss_t)], C.c_int32
    return fn(C.byref(_loss(precision=precision, rows=rows, in_features=cin, classes=classes, ldx=cin, ldw=cin, **kw)))


@pytest.mark.parametrize("rows,cin,classes,blocks", [(1, 4096, 5, 1), (16, 4096, 900, 57), (13, 3696, 9001, 256), (1, 3688, 20011, 256), (16, 4096, 33000, 256), (9, 4088, 12289, 256),
                                                     (1, 2048, 16, 1), (16, 1848, 24601, 512), (2, 2048, 65537, 512)])
def test_streamed_weights(rows, cin, classes, blocks):
    """Four wavefronts take up to 2048 values of a row, eight up to 4096; blocks as many as fit on the card, or as there are groups of 16 classes."""
    assert _path(rows, cin, classes, 1) == _path(rows, cin, classes, 2) == blocks
    if blocks != 57 and blocks > 1:
        assert -(-classes // 16) > blocks, "a block walks more than one group"


@pytest.mark.parametrize("rows,cin,classes", [(16, 4095, 900), (32, 2047, 5003), (33, 517, 40001), (64, 4097, 3001), (1, 7, 130), (48, 1025, 17000)])
def test_weights_as_they_lie(rows, cin, classes):
    assert [_path(rows, cin, classes, p) for p in (0, 1, 2)] == [1, 1, 1]


def test_tiles():
    assert _path(17, 2048, 5000) == 0, "one row more than are streamed"
    assert _path(16, 1024, 5000) == 0 and _path(16, 3000, 5000) == 0, "widths that leave wavefronts without work"
    assert _path(16, 2048, 5000, 0) == 1 and _path(65, 2048, 5000, 0) == 0
    assert _path(16, 2048, 5000, x=AT["x"] + 2) == 0 and _path(16, 2048, 5000, w=AT["w"] + 2) == 1, "off the alignment of 16 bytes"
