"""biq_norm without eps: rows of zeros and rows whose squares' mean has a root that 32 bits do not hold the reciprocal of."""
import numpy as np
import pytest
import torch

import step_util as su
from test_gpu_norm import call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("n", [100, 3000, 40000])
def test_groups_of_zeros_have_scale_0(biq, fmt, group, n):
    """Whatever r is: the header's words.  Rows of zeros, and rows of numbers that are below 2^-100."""
    x = np.zeros((3, n), np.float32)
    x[1], x[2] = 2.0 ** -140, 1
    out = call(biq, x, None, None, "fp32", None, codes=fmt, group=group, eps=0.0)
    assert (out["scales"][:2] == 0).all() and (su.back(out["codes"][:2].float()) == 0).all()
    assert (out["scales"][2] > 0).all()


@pytest.mark.parametrize("n", [1, 100, 3000, 40000])
def test_rows_of_the_least_numbers(biq, n):
    """The norm does not depend on a row's magnitude.  Numbers are whole multiples of 2^-149, exact; three roundings (the root, two products)."""
    rng = np.random.default_rng(n)
    whole = rng.integers(1, 1000, size=(4, n)) * rng.choice([-1, 1], size=(4, n))
    whole[3] = 0
    whole[3, n // 2] = 1
    x = (whole * 2.0 ** -149).astype(np.float32)
    w = (1 + 0.3 * rng.standard_normal(n)).astype(np.float32)
    y = su.back(call(biq, x, None, w, "fp32", "fp32", eps=0.0)["y"])
    want = whole / np.sqrt((whole.astype(np.float64) ** 2).mean(axis=1, keepdims=True)) * w
    assert (np.abs(y - want) <= 2.0 ** -24 * 4 * np.abs(want)).all(), np.max(np.abs(y - want))
