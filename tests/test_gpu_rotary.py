"""Rotary positions against complex numbers in 64 bits; the gradient against differences."""
import math

import numpy as np
import pytest
import torch

import serving_util as su

pytestmark = pytest.mark.gpu
UNIT = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # half a unit of the last place of 1


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


def table(biq, rot, positions, **how):
    turns = biq.biq_rotary_frequencies(rot, **how)
    angles = torch.empty((positions, rot // 2, 2), device="cuda:0")
    biq.biq_rotary_table(turns.to("cuda:0"), angles)
    return angles


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("rows,heads,dim,rot", [(1, 1, 2, 2), (3, 5, 128, 128), (67, 3, 128, 64), (5, 2, 80, 80), (9, 4, 64, 22),
                                                (300, 40, 128, 128), (2, 1, 7, 4), (4, 3, 256, 32), (33, 7, 96, 6)])
def test_against_complex_numbers(biq, typ, interleaved, inverse, rows, heads, dim, rot):
    g = torch.Generator().manual_seed(rows + rot)
    x = torch.randn((rows, heads, dim), generator=g).to(su.TYPES[typ])
    pos = torch.randint(0, 500, (rows,), generator=g, dtype=torch.int32)
    angles = table(biq, rot, 500)
    y = torch.full((rows, heads, dim), float("nan"), dtype=x.dtype, device="cuda:0")
    biq.biq_rotary(x.to("cuda:0"), y, pos.to("cuda:0"), angles, interleaved=interleaved, inverse=inverse)
    a = angles.double().cpu().numpy()[pos.numpy()]
    want = su.turned(x.double().numpy(), a, rot, interleaved, inverse)
    # two products and their sum, each rounded to 32 bits: 2 units of (|a| + |b|); then the output's rounding
    size = np.abs(x.double().numpy()).max()
    assert np.all(np.abs(y.double().cpu().numpy() - want) <= 2 * 2 * size * 2.0 ** -24 + UNIT[typ] * np.abs(want) + 2.0 ** -24)
    assert torch.equal(y.cpu()[..., rot:], x[..., rot:])        # what is not turned comes through
    z = x.to("cuda:0")
    biq.biq_rotary(z, z, pos.to("cuda:0"), angles, interleaved=interleaved, inverse=inverse)
    assert torch.equal(z, y)                                    # in place


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides(biq, typ, interleaved):
    """Queries and keys inside a projection's rows, odd addresses, heads outermost."""
    for lead in (0, 1, 2, 4):
        wide = torch.randn((31 * 9 * 64 + 8,), device="cuda:0").to(su.TYPES[typ])
        x = wide[lead:lead + 31 * 9 * 64].view(31, 9, 64)
        pos = torch.arange(31, dtype=torch.int32, device="cuda:0")
        angles = table(biq, 64, 31)
        want = torch.empty((31, 6, 64), dtype=x.dtype, device="cuda:0")
        biq.biq_rotary(x[:, 1:7].contiguous(), want, pos, angles, interleaved=interleaved)
        out = torch.empty((6, 31, 64), dtype=x.dtype, device="cuda:0").transpose(0, 1)
        biq.biq_rotary(x[:, 1:7], out, pos, angles, interleaved=interleaved)
        assert torch.equal(out, want)
        keep = x.clone()
        biq.biq_rotary(x[:, 1:7], x[:, 1:7], pos, angles, interleaved=interleaved)
        assert torch.equal(x[:, 1:7], want) and torch.equal(x[:, 0], keep[:, 0]) and torch.equal(x[:, 7:], keep[:, 7:])


def test_positions_outside_the_table(biq):
    x = torch.randn((5, 3, 64), device="cuda:0")
    pos = torch.tensor([0, -1, 9, 10, 1 << 30], dtype=torch.int32, device="cuda:0")
    y = torch.zeros_like(x)
    biq.biq_rotary(x, y, pos, table(biq, 32, 10))
    bad = torch.tensor([False, True, False, True, True], device="cuda:0")
    assert torch.isnan(y[bad][..., :32]).all() and torch.equal(y[..., 32:], x[..., 32:]) and torch.isfinite(y[~bad]).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(biq, interleaved):
    """The inverse is the transposed map: against differences of the map, and <g, R x> = <R' g, x>."""
    angles = table(biq, 32, 100)
    pos = torch.tensor([7, 99], dtype=torch.int32, device="cuda:0")
    x, g = torch.randn((2, 2, 40), device="cuda:0"), torch.randn((2, 2, 40), device="cuda:0")

    def forward(x):
        y = torch.empty_like(x)
        biq.biq_rotary(x, y, pos, angles, interleaved=interleaved)
        return y.double()

    dx = torch.empty_like(x)
    biq.biq_rotary(g, dx, pos, angles, interleaved=interleaved, inverse=True)
    h = 2.0 ** -3                                               # (a linear map: the step costs nothing but rounding)
    for d in range(0, 40, 3):
        step = torch.zeros_like(x)
        step[..., d] = h
        diff = (g.double() * (forward(x + step) - forward(x - step))).sum(dim=2) / (2 * h)
        assert (diff - dx[..., d].double()).abs().max() < 1e-5  # 40 terms of magnitude 3 at 2^-24, over the step
    assert abs((g.double() * forward(x)).sum() - (dx.double() * x.double()).sum()) < 1e-5


@pytest.mark.parametrize("rot", [2, 22, 128])
@pytest.mark.parametrize("first", [0, 12345, 2000000000])
def test_table(biq, rot, first):
    turns = biq.biq_rotary_frequencies(rot, 500000.0)
    angles = torch.empty((37, rot // 2, 2), device="cuda:0")
    biq.biq_rotary_table(turns.to("cuda:0"), angles, first=first, amplitude=1.25)
    # the angle's part of a turn is off by 2^-53 of the turns in all at most
    for r in (0, 1, 36):
        for i in {0, rot // 4, rot // 2 - 1}:
            t = (first + r) * turns[i].item()
            angle = 2 * math.pi * (t - round(t))
            slack = 2.0 ** -52 * 2 * math.pi * (abs(t) + 1) + 2.0 ** -23
            assert abs(angles[r, i, 0].item() - 1.25 * math.cos(angle)) < 1.25 * slack
            assert abs(angles[r, i, 1].item() - 1.25 * math.sin(angle)) < 1.25 * slack
