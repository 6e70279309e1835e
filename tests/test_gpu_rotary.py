"""Rotary positions with several axes against the fp64 oracle: forward and gradient, all types, strided and in place."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from paper_2408_10188_amd import binding as B
from paper_2408_10188_amd import paged
from tests.helpers import DEV, nans

pytestmark = pytest.mark.gpu

THETA = 1e6
BF16, F32 = torch.bfloat16, torch.float32

# |error| <= TURN (|a| + |b|) before the result is rounded to its type.  In units of the larger of sine and cosine's own size, 1: the angle is
# kept to 31 bits and then 24 as a number of half turns up to 1 (2^-25 pi = 0.94e-7), sine and cosine of half turns are within 4 ulp (4 * 2^-24), a
# product and a sum of two round three times (3 * 2^-24).  Together 5.1e-7.
TURN = 5.5e-7
HALF_STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def check(y, x, positions, sections, inverse=False):
    a = x.double().cpu().numpy()
    want = orc.rotary(a, positions.cpu().numpy(), sections, THETA, inverse)
    b = np.concatenate(np.split(a, 2, -1)[::-1], -1)
    bound = TURN * (np.abs(a) + np.abs(b))
    bound = bound + HALF_STEP[y.dtype] * (np.abs(want) + bound)
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= bound).all(), float((err / np.maximum(bound, 1e-300)).max())


def inputs(seed, rows, axes, heads, d, dtype, far=1 << 18):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    pos = torch.randint(0, far, (axes, rows), device=DEV, generator=gen, dtype=torch.int32)
    return pos, [torch.randn(rows, h, d, device=DEV, generator=gen).to(dtype) for h in heads]


def sections_of(axes, d):
    return {1: [d // 2], 2: [d // 8, 3 * d // 8], 3: [d // 8, 3 * d // 16, 3 * d // 16], 4: [1, 0, 7, d // 2 - 8]}[axes]


@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("rows,heads,d,axes", [(1, (28, 4), 128, 3), (7, (2, 1), 64, 1), (131, (7, 1), 128, 2), (1000, (4, 2), 64, 4), (3001, (28, 4), 128, 3),
                                               (40000, (1,), 128, 3)])
def test_rotary_against_the_oracle(x_type, y_type, inverse, rows, heads, d, axes):
    pos, x = inputs(rows, rows, axes, heads, d, x_type)
    y = [torch.full(t.shape, float("nan"), dtype=y_type, device=DEV) for t in x]
    B.mmsp_rotary_apply(B.mmsp_rotary_plan(d, THETA, sections_of(axes, d)), rows, pos, rows, [paged.heads_of(t) for t in x], [paged.heads_of(t) for t in y], inverse)
    for a, b in zip(x, y):
        check(b, a, pos, sections_of(axes, d), inverse)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rotary_of_a_projections_slices_in_place(dtype):
    """Q and K inside [rows, Hq + 2 Hkv, d], turned where they lie; V and a padded row of another stride stay as they are."""
    rows, hq, hkv, d = 77, 6, 2, 128
    pos, (full,) = inputs(3, rows, 3, (hq + 2 * hkv + 1,), d, dtype)
    x, before, sections = full[:, :hq + 2 * hkv], full.clone(), sections_of(3, d)
    t = [paged.heads_of(x[:, :hq]), paged.heads_of(x[:, hq:hq + hkv])]
    B.mmsp_rotary_apply(B.mmsp_rotary_plan(d, THETA, sections), rows - 2, pos, rows, t, t)
    check(full[:rows - 2, :hq + hkv], before[:rows - 2, :hq + hkv], pos[:, :rows - 2], sections)
    assert torch.equal(full[rows - 2:], before[rows - 2:]) and torch.equal(full[:, hq + hkv:], before[:, hq + hkv:])


def test_rotary_of_extreme_positions():
    """The whole range of an int32: the oracle's own angle, a product in 64 bits of up to 2^31 rad, is off by 2^-22 there (half a step of 53 bits), far more than
    the kernel's; near and negative ones to the usual bound."""
    d, sections = 128, [64]
    rows = torch.tensor([[0, 1, -1, 5, -262144, 1000003, -1000003]], dtype=torch.int32, device=DEV)
    x = torch.randn(rows.shape[1], 3, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    y = torch.empty_like(x)
    rot = B.mmsp_rotary_plan(d, THETA, sections)
    B.mmsp_rotary_apply(rot, len(x), rows, len(x), [paged.heads_of(x)], [paged.heads_of(y)])
    check(y, x, rows, sections)
    ends = torch.tensor([[2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device=DEV)
    y = torch.empty_like(x[:2])
    B.mmsp_rotary_apply(rot, 2, ends, 2, [paged.heads_of(x[:2])], [paged.heads_of(y)])
    turns = [[(int(p) * int(rot.turns[i])) % 2 ** 64 / 2.0 ** 64 for i in range(64)] for p in ends[0].tolist()]      # exact integers
    angle = 2 * np.pi * np.array(turns)[:, None]
    a, b = np.split(x[:2].double().cpu().numpy(), 2, -1)
    want = np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], -1)
    size = np.tile(np.abs(a) + np.abs(b), 2)
    assert (np.abs(y.double().cpu().numpy() - want) <= TURN * size + 2.0 ** -24 * (np.abs(want) + size)).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_inverse_undoes_and_is_the_gradient(dtype):
    """<dY, R x> = <R^-1 dY, x>: the inverse is the transpose.  And of differences: (R(x + e) - R(x)) . dY / |e| is e . dX."""
    rows, d, sections = 50, 128, sections_of(3, 128)
    pos, (x, dy) = inputs(9, rows, 3, (4, 4), d, dtype)
    rot = B.mmsp_rotary_plan(d, THETA, sections)

    def turn(t, inverse, out=F32):
        y = torch.empty(t.shape, dtype=out, device=DEV)
        B.mmsp_rotary_apply(rot, rows, pos, rows, [paged.heads_of(t)], [paged.heads_of(y)], inverse)
        return y
    x32, dy32 = x.float(), dy.float()
    y, dx = turn(x32, False), turn(dy32, True)
    left, right = (dy32.double() * y.double()).sum(-1), (dx.double() * x32.double()).sum(-1)
    size = (dy32.abs() * (x32.abs() + x32.abs().roll(64, -1))).sum(-1).double() + ((dy32.abs() + dy32.abs().roll(64, -1)) * x32.abs()).sum(-1).double()
    assert bool(((left - right).abs() <= (TURN + 2.0 ** -24) * size).all())
    for i in (0, 5, 63, 64, 100, 127):                     # the map is linear, so a step of 1 has no error of its own
        e = torch.zeros_like(x32)
        e[:, :, i] = 1.0
        slope = ((turn(x32 + e, False).double() - y.double()) * dy32.double()).sum(-1)
        bound = (2 * TURN + 2.0 ** -23) * ((x32.abs() + x32.abs().roll(64, -1) + 1) * dy32.abs()).sum(-1).double() + 2.0 ** -23 * dy32.abs().sum(-1).double() * x32.abs().amax(-1).double()
        assert bool(((slope - dx[:, :, i].double()).abs() <= bound + TURN * (dy32.abs().amax(-1).double() * 2)).all())
    if dtype == BF16:
        check(turn(turn(x, False, BF16), True, BF16), turn(x, False, BF16), pos, sections, True)


def test_rotary_takes_every_row_of_a_long_call():
    """More rows than the chip has threads for at once, three axes that differ, one head."""
    rows, d, sections = 70001, 64, sections_of(3, 64)
    pos, (x,) = inputs(4, rows, 3, (1,), d, BF16)
    y = nans(rows, 1, d, dtype=BF16)
    B.mmsp_rotary_apply(B.mmsp_rotary_plan(d, THETA, sections), rows, pos, rows, [paged.heads_of(x)], [paged.heads_of(y)])
    check(y, x, pos, sections)
