"""biq_attention where values, scales or weights are at the ends of their ranges."""
import numpy as np
import pytest
import torch

import attention_util as au
import serving_util as su

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


def with_values(lens, heads, dim, fmt, seed, magnitudes):
    """A cache whose block b has values of magnitude magnitudes[b % len]."""
    rng = np.random.default_rng(seed)
    c = su.Pages(lens, heads, dim, 64, fmt, rng)
    for s, n in enumerate(lens):
        v = rng.uniform(0.5, 1.0, (n, heads, dim)) * rng.choice([-1.0, 1.0], (n, heads, dim))
        v *= np.array([magnitudes[t // 16 % len(magnitudes)] for t in range(n)])[:, None, None]
        c.append(s, 0, rng.standard_normal((n, heads, dim)).astype(np.float32).astype(np.float64), v.astype(np.float32).astype(np.float64))
    return c


MAGNITUDES = [[2.0 ** -99.5], [2.0 ** -98], [2.0 ** -95], [2.0 ** -92], [2.0 ** -88], [2.0 ** -84], [2.0 ** -60], [2.0 ** -97, 2.0 ** -91, 2.0 ** -85],
              [2.0 ** -98, 2.0 ** -70], [2.0 ** -98, 1.0], [2.0 ** 100], [0.0, 2.0 ** -98], [0.0]]


@pytest.mark.parametrize("magnitudes", MAGNITUDES)
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_values_of_any_magnitude(biq, typ, fmt, magnitudes):
    """Errors stay relative to the largest value, whatever it is (a block is held from 2^-100 on, so its scale is down to 2^-108)."""
    pages = with_values([300, 90], 2, 64, fmt, 1, magnitudes)
    for counts in ([1, 1], [40, 3]):                            # few rows
        au.check(biq, pages, counts, au.rows_like(counts, 4, 64, typ, 2), typ)
    pages = with_values([160, 100], 16, 32, fmt, 2, magnitudes)
    counts = [160, 90]                                          # many
    au.check(biq, pages, counts, au.rows_like(counts, 128, 32, typ, 3), typ, sample=[0, 1, 17, 70, 89, 159])


@pytest.mark.parametrize("magnitudes", [[0.0, 2.0 ** 100], [2.0 ** 100, 2.0 ** -98]])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_nothing_beside_large_values(biq, typ, magnitudes):
    """Rows whose window has blocks of either kind, and of one kind only."""
    pages = with_values([300, 90], 2, 64, "int8", 1, magnitudes)
    for counts in ([1, 1], [40, 3]):
        for window in (0, 16, 5):
            au.check(biq, pages, counts, au.rows_like(counts, 4, 64, typ, 2), typ, window=window)


def constant(length, low, k_low, k_high, value):
    """One head of 16: keys k_low for the first `low` tokens, k_high for the others, values value(tokens); rows of ones see
    16 k_low scale and 16 k_high scale."""
    c = su.Pages([length], 1, 16, 256, "int8", np.random.default_rng(1))
    k = np.where(np.arange(length) < low, k_low, k_high)[:, None, None] * np.ones((1, 1, 16))
    v = value(np.arange(length))[:, None, None] * np.ones((1, 1, 16))
    c.append(0, 0, k, v)
    return c


def test_many_tokens_whose_values_are_zeros(biq):
    """The sum of the weights stays a number although no value bounds the reference: 40000 tokens, 7.5 doublings above the first ones."""
    up = 7.5 * np.log(2) / 16
    pages = constant(40000, 256, 0.0, up, lambda t: 0.0 * t)
    q = torch.ones((1, 1, 16))
    out, _ = au.check(biq, pages, [1], q, "fp32", scale=1.0, max_len=64)       # one workgroup walks through all tokens
    assert (out == 0).all()
    au.check(biq, pages, [1], q.bfloat16(), "bf16", scale=1.0, max_len=64)
    q = torch.ones((3000, 16, 16))                              # one wave does
    au.check(biq, pages, [3000], q, "fp32", scale=1.0, sample=[0, 1499, 2999])
    au.check(biq, pages, [3000], q.bfloat16(), "bf16", scale=1.0, sample=[0, 1499, 2999])


@pytest.mark.parametrize("doublings", [26.0, 31.4, 33.0])
def test_a_long_tail_behind_one_large_weight(biq, doublings):
    """130984 weights of 2^-31.4 of the first one are 5e-5 of the sum, which a 32-bit output shows: the first token's value is 0, the
    others' are 1, so the output is the tail's share.  Weights are lost below 2^-38 of the largest; the tail's sum is off by a unit for every
    step of 64 (2047 of 2^-24) and by the weights' own errors (1e-5), 2^-10 of it in all at most."""
    up = doublings * np.log(2) / 32
    length = 131000
    pages = constant(length, 16, up, -up, lambda t: np.where(t == 0, 0.0, 1.0))
    for s in range(1, 16):                                      # of the first block one token only has the large score
        pages.store[pages.table[0, 0], s * 16:(s + 1) * 16] = np.int8(-127).view(np.uint8)
    q = torch.ones((2900, 16, 16))
    for rows, how in ((q, {}), (q[:1, :1].contiguous(), dict(max_len=64))):    # one wave; one workgroup
        out, _ = au.check(biq, pages, [rows.shape[0]], rows, "fp32", scale=1.0, sample=[0, 1450, 2899], **how)
        k, v = (torch.from_numpy(x) for x in pages.values(0))
        want, _, _, _ = au.softmax64(rows[-1:].double(), k, v, 1.0, torch.tensor([length - 1]), True, 0)
        assert ((out[-1:] - want).abs() <= length * 2.0 ** -38 + 2.0 ** -10 * want).all(), (out[-1, 0, 0].item(), want[0, 0, 0].item())
