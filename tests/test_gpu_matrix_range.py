"""Orthogonalised updates at the ends of their range: long sides."""
import pytest

from tests.test_gpu_matrix import env, exactly, update  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(32, 131072), (131072, 32), (16, 262144), (8, 1 << 20), (4, 1 << 19), (1 << 19, 4), (1, 1 << 20), (33, 40000),
                                       (300, 20000), (20000, 300), (2816, 9000), (2900, 9000), (4100, 4200)])
def test_long_sums_keep_the_documented_accuracy(env, rows, cols):
    """The numbers that the header gives: HALF within 4e-3 (fewer than eight rows or columns: 1e-2) and SINGLE within 2e-6 (5e-6) for well
    conditioned updates, 3e-2 and 2e-5 for one direction and one percent of noise.  An update of +-1 is the hardest one: its
    Gram matrix's diagonal adds up equal squares, whose roundings all go the same way."""
    B, torch = env
    gen = torch.Generator(device="cuda").manual_seed(2)
    noise = torch.randn(rows, cols, generator=gen, device="cuda")
    thin = torch.randn(rows, 1, generator=gen, device="cuda") * torch.randn(1, cols, generator=gen, device="cuda") + 0.01 * noise
    well = (1e-2, 5e-6) if min(rows, cols) < 8 else (4e-3, 2e-6)
    for what, g, allowed in (("noise", noise, well), ("update", update(torch, rows, cols, 1), well), ("signs", 1.3 * noise.sign(), well),
                             ("thin", thin, (3e-2, 2e-5))):
        want = exactly(g.double())
        for products in (B.PRODUCTS_HALF, B.PRODUCTS_SINGLE):
            out = torch.empty_like(g)
            plan = B.MatrixPlan(rows, cols, products=products)
            plan.fo_orthogonalize([g], [out])
            off = float((out.double() - want).norm() / want.norm())
            print(f"{rows} x {cols} {what}: off by {off:.2e}, allowed {allowed[products]:.1e}", flush=True)
            assert off <= allowed[products]
            plan.close()


def test_outputs_that_meet_anything_else_are_refused(env):
    """Every way in which rows can lie in other rows, and the ways in which they only look as if they did."""
    B, torch = env
    rows, cols = 8, 12
    plan = B.MatrixPlan(rows, cols, count=2)

    def at(flat, first, ld):
        return flat.as_strided((rows, cols), (ld, 1), first)

    def refused(g, out):
        with pytest.raises(B.FoError) as e:
            plan.fo_orthogonalize(g, out)
        assert e.value.code == B.EINVAL

    flat, other = torch.randn(2000, device="cuda"), torch.zeros(2000, device="cuda")
    before = flat.clone()
    g = [at(flat, 0, 24), at(flat, 500, 24)]
    o = at(other, 0, 24)
    for first in (24, 1, 23, 24 * 7, 24 * 7 + 11, 500 - 11, 500 + 24 * 8 - 13, 512 - 1):   # rows or a part of one further on, or before it
        refused(g, [at(flat, first, 24), o])
        refused(g, [o, at(flat, first, 24)])
    refused(g, [at(other, 0, 24), at(other, 11, 24)])                                      # outputs
    refused(g, [at(other, 0, 24), at(other, 24 * 7 + 11, 24)])
    for first, ld in ((0, 25), (13, 23), (24 * 7 + 11, 13), (500 - 7 * 31, 31), (24, 48)):  # another stride
        refused(g, [at(flat, first, ld), at(other, first, ld)])
    torch.cuda.synchronize()
    assert torch.equal(flat, before) and not bool(other.any())
    alone = [at(torch.zeros(200, device="cuda"), 0, 24 if k else 12) for k in (0, 0)]
    plan.fo_orthogonalize(g, alone)
    for outs in ([at(flat, 12, 24), at(flat, 512, 24)], [at(flat, 24 * 7 + 12, 24), at(flat, 500 + 24 * 7 + 12, 24)],
                 [at(flat, 12, 48), at(flat, 1000, 48)]):                                  # between the rows, behind the last one
        flat.copy_(before)
        plan.fo_orthogonalize(g, outs)
        assert torch.equal(outs[0], alone[0]) and torch.equal(outs[1], alone[1])
        assert torch.equal(g[0], at(before, 0, 24)) and torch.equal(g[1], at(before, 500, 24))
    one = B.MatrixPlan(1, cols)
    with pytest.raises(B.FoError):
        one.fo_orthogonalize([flat[None, 0:12]], [flat[None, 11:23]])
    one.fo_orthogonalize([flat[None, 0:12]], [flat[None, 12:24]])
