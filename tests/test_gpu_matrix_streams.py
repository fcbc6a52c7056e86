"""The matrix operators on streams other than the one that their memory is of."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_plan_may_be_dropped_while_another_stream_uses_it():
    """Its workspace holds the tables that the kernels read: the memory must not go to the next allocation before they have."""
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(1)
    g = torch.randn(200 * 300, generator=gen, device="cuda")
    want = B.Orthogonalizer([(200, 300)]).orthogonalize(g)
    torch.cuda.synchronize()
    plan = B.Orthogonalizer([(200, 300)])
    side, out = torch.cuda.Stream(), torch.empty_like(g)
    size, where = plan.workspace.numel(), plan.workspace.data_ptr()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)  # (some 10 ms)
        plan.orthogonalize(g, out)
    del plan
    others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert all(o.data_ptr() != where for o in others)
    for o in others:
        o.fill_(255)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_a_new_result_is_zero_between_the_matrices():
    """Not what the allocation before it left there."""
    import torch
    from paper_2105_00619_amd import binding as B
    for mats, n in (([(3, 10, 20, 50), (777, 33, 65, 71)], 777 + 33 * 71), ([(8, 9)], 200)):
        p = B.Orthogonalizer(mats)
        g = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
        inside = torch.zeros(n, dtype=torch.bool, device="cuda")
        for m in mats:
            off, r, c, ld = m if len(m) == 4 else (0, *m, m[1])
            torch.as_strided(inside, (r, c), (ld, 1), off).fill_(True)
        for _ in range(3):
            junk = torch.full((n,), float("nan"), device="cuda")
            del junk
            o = p.orthogonalize(g)
            assert bool((o[~inside] == 0).all()) and bool((o[inside] != 0).all())
            del o
