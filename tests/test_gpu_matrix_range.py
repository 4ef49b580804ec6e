"""Orthogonalised updates at the ends of their range: long sides, overlaps, values that are no numbers, few steps and many."""
import pytest

from tests.test_gpu_matrix import COEFFICIENTS, check, env, exactly, update  # noqa: F401

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


BOTH_PATHS = [(40, 70), (70, 40), (1, 9), (128, 128), (150, 200), (200, 150), (300, 1), (129, 129)]  # in one workgroup up to 128 x 128


@pytest.mark.parametrize("dtype,single", [("float32", True), ("float32", False), ("bfloat16", False), ("float16", True)])
@pytest.mark.parametrize("rows,cols", BOTH_PATHS)
def test_any_magnitude_zero_and_no_numbers_side_by_side(env, rows, cols, dtype, single):
    """What one matrix of a call holds is its own affair, on either path: a power of two changes no bit, zeros stay zeros, and an infinity
    or a NaN spoils its own matrix everywhere and no other."""
    B, torch = env
    dt = getattr(torch, dtype)
    kw = dict(dtype=dt, products=B.PRODUCTS_SINGLE if single else B.PRODUCTS_HALF)
    up, down = (2.0 ** 9, 1.0) if dtype == "float16" else (2.0 ** 120, 2.0 ** -100)       # (fp16 has no room below)
    g = torch.stack([update(torch, rows, cols, 1).to(dt).float() * f for f in (1, up, down, 0, 1, 1, 1, 1)]).to(dt)
    g[4, rows // 2, cols // 2], g[5, 0, 0], g[6, rows - 1, cols - 1] = float("nan"), float("inf"), -float("inf")
    out = torch.empty_like(g)
    B.MatrixPlan(rows, cols, count=8, **kw).fo_orthogonalize(g, out)
    assert bool(out[0].isfinite().all()) and bool(out[0].any())
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2]) and torch.equal(out[0], out[7]) and not bool(out[3].any())
    assert bool(out[4:7].isnan().all())


@pytest.mark.parametrize("nesterov", (False, True))
@pytest.mark.parametrize("rows,cols", BOTH_PATHS)
def test_steps_with_zeros_and_no_numbers_side_by_side(env, rows, cols, nesterov):
    """A step of a normal gradient beside one of zeros (parameters decay, nothing else), zeros with a momentum, a NaN and an infinity."""
    B, torch = env
    kw = dict(nesterov=nesterov, scale=2.0, decay=0.1)
    g = torch.stack([update(torch, rows, cols, k) for k in range(5)])
    m = torch.stack([update(torch, rows, cols, 10 + k) for k in range(5)])
    x = torch.stack([update(torch, rows, cols, 20 + k) * 20 for k in range(5)])
    g[1:3] = 0
    m[1] = 0
    g[3, rows - 1, 0], g[4, 0, cols - 1] = float("nan"), -float("inf")
    m1, x1 = m.clone(), x.clone()
    B.MatrixPlan(rows, cols, count=5).fo_matrix_step(g, m1, x1, 0.02, **kw)
    one = B.MatrixPlan(rows, cols)
    for k in (0, 2):
        mk, xk = m[k].clone(), x[k].clone()
        one.fo_matrix_step([g[k]], [mk], [xk], 0.02, **kw)
        assert torch.equal(m1[k], mk) and bool(x1[k].isfinite().all())
        # (one matrix may take other tiles, whose sums are in another order)
        assert float((x1[k].double() - xk.double()).norm()) <= 1e-5 * float((xk.double() - x[k].double()).norm())
    f32 = torch.tensor
    keep = f32(1.0 - float(f32(0.02, dtype=torch.float32)) * float(f32(0.1, dtype=torch.float32)), dtype=torch.float32).cuda()
    assert not bool(m1[1].any()) and torch.equal(x1[1], x[1] * keep)
    for k, bad in ((3, g[3].isnan()), (4, g[4].isinf())):
        assert torch.equal(m1[k].isfinite(), ~bad) and bool(x1[k].isnan().all())


@pytest.mark.parametrize("rows,cols", [(100, 70), (70, 100), (128, 128), (1, 50), (33, 31), (150, 100)])
def test_steps_and_coefficients_of_either_orientation(env, rows, cols):
    B, torch = env
    g = update(torch, rows, cols, 1)
    for steps, k in ((1, COEFFICIENTS), (2, COEFFICIENTS), (3, (2.0, -1.5, 0.5)), (12, (1.875, -1.25, 0.375)), (16, (1.5, -0.5, 0.0))):
        for single in (False, True):
            plan = B.MatrixPlan(rows, cols, products=int(single), steps=steps, coefficients=k)
            out = torch.empty_like(g)
            plan.fo_orthogonalize([g], [out])
            check(torch, out, g, single, f"{steps} steps", steps=steps, coefficients=k)


@pytest.mark.parametrize("dtype,single", [("float32", True), ("bfloat16", True), ("float16", False)])
@pytest.mark.parametrize("rows,cols", [(4100, 4200), (4200, 4100), (40, 9000), (9000, 40)])
def test_steps_of_long_sums_take_what_orthogonalize_gives(env, rows, cols, dtype, single):
    """x <- keep x - by O for the O of fo_orthogonalize: three roundings of fp32 of either term, and half a step of the type."""
    B, torch = env
    dt = getattr(torch, dtype)
    products = B.PRODUCTS_SINGLE if single else B.PRODUCTS_HALF
    g, o = update(torch, rows, cols, 3), torch.empty(rows, cols, device="cuda")
    B.MatrixPlan(rows, cols, products=products).fo_orthogonalize([g], [o])
    m, x = torch.zeros_like(g), (update(torch, rows, cols, 4) * 20).to(dt)
    x0 = x.double()
    B.MatrixPlan(rows, cols, dtype=dt, products=products).fo_matrix_step([g], [m], [x], 0.5, mu=0.0, nesterov=False, scale=0.25, decay=0.25)
    assert torch.equal(m, g)
    keep, by = 0.875, 0.125
    allowed = (3 * 2.0 ** -24 + torch.finfo(dt).eps / 2) * 1.001 * (keep * x0.abs() + by * o.double().abs()) + 2.0 ** -25
    assert bool(((x.double() - (keep * x0 - by * o.double())).abs() <= allowed).all())
