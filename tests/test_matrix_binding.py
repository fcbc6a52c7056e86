"""The Python side of the matrix operators without a GPU: what it asks of torch and of the library."""
import contextlib
import os
import types

import pytest

from paper_2105_00619_amd import binding as B


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(B.LIB_PATH):
        from paper_2105_00619_amd import build
        build.build(verbose=False)


class _Bound(B.Orthogonalizer):
    """An Orthogonalizer whose device is made up: stream numbers, a workspace that notes the streams it is told of, a library that does nothing."""

    def __init__(self, home):
        self.stream, self.capturing, self.told, self.home = home, False, [], home
        cuda = types.SimpleNamespace(
            current_stream=lambda device: types.SimpleNamespace(cuda_stream=self.stream),
            is_current_stream_capturing=lambda: self.capturing, device=lambda d: contextlib.nullcontext())
        self.torch = types.SimpleNamespace(cuda=cuda)
        self.device, self.handle = "cuda:0", None
        self.workspace = types.SimpleNamespace(record_stream=lambda s: self.told.append(s.cuda_stream))
        self.calls = []
        self.lib = types.SimpleNamespace(optorch_orthogonalize=lambda *a: self.calls.append(a[-1]) or B.OK,
                                         optorch_muon_update=lambda *a: self.calls.append(a[-1]) or B.OK)

    def _flat(self, name, t, dtypes=None):
        return 0


def test_the_allocator_is_told_of_every_stream_that_uses_a_workspace():
    v = types.SimpleNamespace(data_ptr=lambda: 1 << 20)
    o = _Bound(home=7)
    o.orthogonalize(v, v)
    assert o.told == [] and o.calls == [7]
    o.stream = 9
    o.orthogonalize(v, v)
    assert o.told == [9] and o.calls == [7, 9]
    o.stream = 11
    o.muon_update(v, v, v, lr=0.1)
    assert o.told == [9, 11] and o.calls == [7, 9, 11]
    o.capturing = True  # (nothing runs; the graph's user keeps the object)
    o.orthogonalize(v, v)
    assert o.told == [9, 11]


def test_no_steps_are_five_and_so_are_their_coefficients(monkeypatch):
    """The library takes steps <= 0 for five and reads three coefficients of each."""
    seen = []

    def create(arr, n, cfg, out):
        cfg = cfg._obj
        seen.append((cfg.steps, [cfg.coefficients[i] for i in range(3 * cfg.steps)]))
        return B.OK

    monkeypatch.setattr(B, "load_library", lambda: types.SimpleNamespace(
        optorch_ortho_create=create, optorch_ortho_query=lambda *a: B.OK, optorch_ortho_destroy=lambda h: None))
    for steps in (0, -3, 5):
        B.OrthoPlan([(4, 4)], steps=steps, coefficients=(2.0, -1.5, 0.5))
        B.OrthoPlan([(4, 4)], steps=steps, coefficients=[(2.0, -1.5, 0.5)] * 5)
    assert seen == [(5, [2.0, -1.5, 0.5] * 5)] * 6


def test_sizes_beyond_their_c_fields_are_refused():
    """2^32 + 4 is not 4."""
    import torch
    for m in ((2 ** 32 + 4, 4), (4, 2 ** 32 + 4), (0, 4, 2 ** 31, 2 ** 31), (0, -2 ** 32 + 4, 4, 4)):
        with pytest.raises(ValueError, match="too large"):
            B.OrthoPlan([m])
    x = types.SimpleNamespace(is_cuda=True, dtype=torch.bfloat16)
    for cin, cout, name in ((2 ** 32 + 8, 8, "in_features"), (8, 2 ** 32 + 8, "out_features")):
        with pytest.raises(ValueError, match=name):
            B._linear_args(x, "none", 0, cin, cout)
    assert B._linear_args(x, "none", 0, 8, 16).out_features == 16


def test_weights_are_updated_after_they_were_set():
    from paper_2105_00619_amd import workloads as W
    p = B.SeqPlan.from_workload(W.config(3))
    lib = B.load_library()
    src = (B.C.c_float * p.param_count)()
    assert lib.optorch_seq_update_params(p.handle, src, p.param_count, 0) == B.E_ORDER
    assert lib.optorch_seq_update_params(None, src, p.param_count, 0) == B.E_INVALID


def test_the_flag_of_skipped_updates_is_on_the_plans_device():
    import torch
    v = types.SimpleNamespace(data_ptr=lambda: 1 << 20)
    o = _Bound(home=7)
    o.index, o.torch.int32 = 1, torch.int32
    flag = lambda device, cuda=True: types.SimpleNamespace(  # noqa: E731
        dtype=torch.int32, numel=lambda: 1, is_cuda=cuda, device=types.SimpleNamespace(index=device), data_ptr=lambda: 1 << 20)
    o.muon_update(v, v, v, lr=0.1, skipped=flag(1))
    assert o.calls == [7]
    for bad in (flag(0), flag(2), flag(1, cuda=False)):
        with pytest.raises(TypeError, match="skipped"):
            o.muon_update(v, v, v, lr=0.1, skipped=bad)
    assert o.calls == [7]
