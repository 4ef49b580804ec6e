"""8-bit rows at the ends of their range: finite values whose transform leaves fp32's, codes that saturate."""
import numpy as np
import pytest

from tests.row_codes import off_from_definition
from tests.test_gpu_rows import CASES, ROUND, SEED, TYPES, _check_codes, _dithers, _flattened, _matrix, _signs, env  # noqa: F401

pytestmark = pytest.mark.gpu


def _rows(torch, rows, length, dtype, seed):
    """Rows with values up to 3.3e38, of which the first is ordinary."""
    x = torch.randn(rows, length, generator=torch.Generator().manual_seed(seed)).clamp_(-3, 3)
    x[1:] *= 1.1e38
    return x.to(dtype).cuda()


def _encode(B, torch, x, block, turned, dither):
    rows, length = x.shape
    q = torch.empty(rows, B.fo_rows_stride(length, block), dtype=torch.int8, device="cuda")
    s = torch.empty(rows, device="cuda")
    B.fo_rows_encode(x.t().contiguous() if turned else x, q, s, block_log2=block, seed=SEED, rnd=ROUND, party=11, transposed=turned,
                     dither=B.DITHER_UNIFORM if dither else B.DITHER_NONE)
    return q, s


@pytest.mark.parametrize("dtype", ("float32", "bfloat16"))
@pytest.mark.parametrize("length,block,dither", [(64, 6, False), (300, 7, True), (2500, 8, False), (8000, 9, True), (16384, 10, False), (20000, 10, False),
                                                 (20000, 6, True), (300, 0, False)])
def test_rows_whose_transform_leaves_the_range(env, oracle, length, block, dither, dtype):
    """Sums of 2^block finite values are up to 2^block times larger than the largest float; their codes and amplitudes are not."""
    B, torch = env
    rows = 4
    x = _rows(torch, rows, length, getattr(torch, dtype), length)
    stride = B.fo_rows_stride(length, block)
    u = _dithers(oracle, rows, stride, 11) if dither else np.zeros((rows, stride))
    found = [_encode(B, torch, x, block, turned, dither) for turned in (False, True)]
    for q, s in found:
        _check_codes(q.cpu().numpy().astype(np.float64), s.double().cpu().numpy(), x.double().cpu().numpy(), stride, block,
                     _signs(oracle, stride) if block else None, u)
    assert torch.equal(found[0][0], found[1][0]) and torch.equal(found[0][1], found[1][1])


@pytest.mark.parametrize("turned", (False, True))
def test_their_neighbours_keep_their_codes(env, turned):
    """Rows that a workgroup takes one after the other, columns of one tile: ordinary ones, ones that leave the range, an infinity, a NaN."""
    B, torch = env
    rows = (1 << 14) + 70
    x = torch.randn(rows, 100, generator=torch.Generator().manual_seed(4)).cuda()
    alone = _encode(B, torch, x, 7, turned, False)
    y = x.clone()
    kind = torch.arange(rows, device="cuda") % 7
    y[kind == 1] *= 2.0 ** 125
    y[kind == 3, 50] = float("inf")
    y[kind == 4, 99] = float("nan")
    q, s = _encode(B, torch, y, 7, turned, False)
    bad = (kind == 3) | (kind == 4)
    assert bool(s[bad].isnan().all()) and not bool(q[bad].any())
    assert torch.equal(q[~bad], alone[0][~bad])                                           # (a power of two changes no code)
    assert torch.equal(s[(kind != 1) & ~bad], alone[1][(kind != 1) & ~bad])
    want = alone[1][kind == 1].double() * 2.0 ** 125
    assert bool(((s[kind == 1].double() - want).abs() <= 2.0 ** -23 * want).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,length,block,pad,dither", CASES)
def test_saturated_codes_too(env, oracle, rows, length, block, pad, dither, dtype):
    """Every code against its definition, those at the ends of the range with their sign and on ragged tails."""
    B, torch = env
    x = _matrix(torch, rows, length, getattr(torch, dtype), pad, rows + length + 1)
    stride = B.fo_rows_stride(length, block)
    y, total = _flattened(x.double().cpu().numpy(), stride, block, _signs(oracle, stride) if block else None)
    u = _dithers(oracle, rows, stride, 11) if dither else np.zeros((rows, stride))
    for turned in (False, True):
        q, s = _encode(B, torch, x, block, turned, dither)
        q = q.cpu().numpy().astype(np.float64)
        assert np.all(off_from_definition(q, y, total, u, block) <= 0)
        assert np.all(np.abs(q).max(axis=1)[np.abs(y).max(axis=1) > 0] == 127)
