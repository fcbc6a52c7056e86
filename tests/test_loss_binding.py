"""The Python side of the losses without a GPU: sizes that the C fields do not hold."""
import pytest

from paper_2105_00619_amd import binding as B


def test_a_teachers_entries_that_their_c_field_does_not_hold():
    """2^32 + 5 entries a row were five."""
    torch = pytest.importorskip("torch")
    a = B.optorch_softmax_loss_t()
    a.rows = 1
    meta = lambda *s, dtype: torch.empty(*s, dtype=dtype, device="meta")  # noqa: E731
    x = meta(1, 8, dtype=torch.float32)
    n = (1 << 32) + 5
    with pytest.raises(ValueError, match="top"):
        B._teacher(a, x, meta(1, n, dtype=torch.int32), meta(1, n, dtype=torch.bfloat16), 1.0)
    B._teacher(a, x, meta(1, 5, dtype=torch.int32), meta(1, 5, dtype=torch.bfloat16), 1.0)
    assert a.top == 5
