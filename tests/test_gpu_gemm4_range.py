"""biq_gemm4 where inputs or weights' scales are near the ends of 32 bits and the products are not: whatever the number of vectors."""
import numpy as np
import pytest
import torch

import step_util as su
from test_gpu_gemm4 import call, check, packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


def weights(m, n, group, scale, seed):
    """Codes that are mostly large and of one sign, scales about `scale`."""
    rng = np.random.default_rng(seed)
    return rng.integers(4, 8, size=(m, n)).astype(np.int8), su.bf16(rng.uniform(1, 2, size=(m, su.groups(n, group))) * scale)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("batch", [1, 5, 16, 20, 40, 64])
@pytest.mark.parametrize("big,scale", [(1e36, 1e-3), (1e38, 1e-6), (1e38, 1e-30), (1e-25, 2.0 ** 98), (1e-30, 2.0 ** 100), (1e25, 1e-28)])
def test_large_inputs_and_small_scales(biq, kind, group, batch, big, scale):
    codes, scales = weights(70, 300, group, scale, batch)
    x = np.random.default_rng(group).uniform(0.5, 1, size=(batch, 300)) * big
    t = su.to(x.astype(np.float32), kind)
    y = call(biq, packed(biq, codes, scales, group), t, 70, group, "fp32")
    assert torch.isfinite(y).all()
    check(y, codes, scales, su.back(t), group, "fp32")


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("group,x_group", [(32, 0), (128, 128), (128, 32), (64, 32), (32, 64)])
@pytest.mark.parametrize("batch", [1, 16, 20, 64])
@pytest.mark.parametrize("x_scale,scale", [(1e35, 1e-6), (3e38, 1e-20), (1e-30, 2.0 ** 100)])
def test_large_scales_of_codes(biq, kind, group, x_group, batch, x_scale, scale):
    codes, scales = weights(40, 300, group, scale, batch)
    rng = np.random.default_rng(batch)
    c = torch.from_numpy(rng.integers(60, 128, size=(batch, 300))).to(torch.int8 if kind == "int8" else torch.float8_e4m3fn)
    s = (rng.uniform(0.5, 1, size=(batch, su.groups(300, x_group))) * x_scale).astype(np.float32)
    y = call(biq, packed(biq, codes, scales, group), c.to("cuda:0"), 40, group, "fp32", torch.from_numpy(s).to("cuda:0"), x_group)
    assert torch.isfinite(y).all()
    check(y, codes, scales, c.double().numpy() * su.spread(s.astype(np.float64), 300, x_group), group, "fp32")
