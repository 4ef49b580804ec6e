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
