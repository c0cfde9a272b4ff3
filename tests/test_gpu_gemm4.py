"""biq_gemm4 and its layout against 64 bits."""
import numpy as np
import pytest
import torch

import step_util as su

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


def packed(biq, codes, scales, group):
    m, n = codes.shape
    out = torch.full((biq.biq_packed4_bytes(m, n, group),), 0xa5, dtype=torch.uint8, device="cuda:0")
    biq.biq_pack4(torch.from_numpy(codes).to("cuda:0"), torch.from_numpy(scales).to("cuda:0"), out, m, n, group)
    return out


def weights(m, n, group, seed):
    rng = np.random.default_rng(seed)
    return rng.integers(-8, 8, size=(m, n)).astype(np.int8), su.bf16(rng.uniform(0.01, 0.05, size=(m, su.groups(n, group))))


def inputs(batch, n, kind, x_group, seed):
    """Tensor, scales (or None), and the values in 64 bits."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((batch, n)) * np.exp(rng.standard_normal(n))
    if kind not in ("int8", "fp8"):
        t = su.to(x.astype(np.float32), kind)
        return t, None, su.back(t)
    c = torch.from_numpy(np.clip(np.rint(x * 20), -128, 127)).to(torch.int8) if kind == "int8" else torch.from_numpy(x).to(torch.float8_e4m3fn)
    s = rng.uniform(0.5, 2, size=(batch, su.groups(n, x_group))).astype(np.float32)
    return c.to("cuda:0"), torch.from_numpy(s).to("cuda:0"), c.double().numpy() * su.spread(s.astype(np.float64), n, x_group)


def call(biq, w, x, m, group, y_type, x_scales=None, x_group=0, pad=0):
    y = torch.full((x.shape[0], m + pad), float("nan"), dtype=su.TYPES[y_type], device="cuda:0")
    ws = torch.full((max(16, biq.biq_gemm4_workspace_bytes(w, x, y[:, :m], group, x_scales=x_scales, x_group=x_group)),), 0xff, dtype=torch.uint8,
                    device="cuda:0")
    biq.biq_gemm4(w, x, y[:, :m], group, x_scales=x_scales, x_group=x_group, workspace=ws)
    torch.cuda.synchronize()
    assert pad == 0 or torch.isnan(y[:, m:]).all()
    return y[:, :m]


def check(got, codes, scales, x, group, y_type):
    """X keeps 22 bits (2^-22 of an element; of the largest of 128 at worst 2^-39, within the next term); a product's 32 elements are added in at most
    32 roundings, 8 products (two terms) follow one another, then the groups of a row, n / 32 at most, and 8 waves: of the sum of magnitudes a
    share of 2^-24 (4 + 32 * 8 + n / 32 + 8) at the very worst.  Roundings that fall either way stay far below: the norm of the
    differences is held to 2^-21 of that of the sums of magnitudes."""
    w = codes.astype(np.float64) * su.spread(scales.astype(np.float64), codes.shape[1], group)
    want, size = x @ w.T, np.abs(x) @ np.abs(w).T
    off = np.abs(su.back(got) - want)
    own = su.HALF[y_type] * np.abs(want) * (1 + 2.0 ** -8) + 2.0 ** -25
    assert (off <= 2.0 ** -24 * (268 + codes.shape[1] / 32) * size + own).all()
    assert np.linalg.norm(np.maximum(off - own, 0)) <= 2.0 ** -21 * np.linalg.norm(size)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n", [(1, 1), (15, 31), (16, 128), (17, 129), (40, 300), (33, 4097)])
def test_layout(biq, group, m, n):
    codes, scales = weights(m, n, group, m + n)
    w = packed(biq, codes, scales, group)
    out = torch.full((m, n + 3), float("nan"), device="cuda:0")
    biq.biq_unpack4(w, out[:, :n], m, n, group)
    assert np.array_equal(su.back(out[:, :n]), codes.astype(np.float64) * su.spread(scales.astype(np.float64), n, group))
    assert torch.isnan(out[:, n:]).all()


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n", [(1, 1), (18, 77), (33, 513)])
def test_quantizer(biq, typ, group, m, n):
    rng = np.random.default_rng(m + n)
    w = rng.standard_normal((m, n)).astype(np.float32)
    if m > 4:
        w[1], w[2, :5], w[3] = 0, 1e-31 if typ != "fp16" else 0, 0
        w[3, 0] = 5
        w[4, n - 1] = np.inf
    t = su.to(w, typ)
    w = su.back(t).astype(np.float32)
    out = torch.full((biq.biq_packed4_bytes(m, n, group),), 0xa5, dtype=torch.uint8, device="cuda:0")
    wide = torch.full((m, n + 5), float("nan"), dtype=t.dtype, device="cuda:0")[:, :n]
    wide.copy_(t)
    biq.biq_quantize4(wide, out, m, n, group)
    codes, scales = su.quantized4(w, group)
    assert torch.equal(out, packed(biq, codes, scales, group))


@pytest.mark.parametrize("kind,x_group", [("fp32", 0), ("bf16", 0), ("fp16", 0), ("int8", 0), ("int8", 32), ("int8", 128), ("fp8", 64), ("fp8", 0)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,batch", [(1, 1, 1), (16, 128, 1), (17, 127, 2), (50, 129, 3), (100, 1000, 15), (130, 700, 16), (64, 500, 17), (35, 4100, 33),
                                       (20, 260, 64), (19, 300, 65), (9, 3, 40), (30, 7, 2), (31, 8, 33), (33, 13, 20), (5, 263, 18), (48, 140, 130), (3000, 513, 5), (40000, 130, 2)])
def test_products(biq, kind, x_group, group, m, n, batch):
    codes, scales = weights(m, n, group, m + n)
    x, x_scales, values = inputs(batch, n, kind, x_group, batch)
    y_type = {"fp32": "fp32", "bf16": "bf16", "fp16": "fp16", "int8": "fp32", "fp8": "bf16"}[kind]
    check(call(biq, packed(biq, codes, scales, group), x, m, group, y_type, x_scales, x_group, pad=m % 3), codes, scales, values, group, y_type)


@pytest.mark.parametrize("kind", ["fp32", "bf16", "int8"])
@pytest.mark.parametrize("m,n,batch", [(300, 16384, 1), (64, 16384, 9), (100, 40000, 3), (48, 20000, 40)])
def test_long_rows(biq, kind, m, n, batch):
    codes, scales = weights(m, n, 128, n)
    x, x_scales, values = inputs(batch, n, kind, 128, n)
    check(call(biq, packed(biq, codes, scales, 128), x, m, 128, "fp32", x_scales, 128 if kind == "int8" else 0), codes, scales, values, 128, "fp32")


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("m,n,batch", [(70, 333, 1), (70, 4096, 3), (70, 333, 20), (500, 1111, 64)])
def test_whole_numbers_are_exact(biq, kind, m, n, batch):
    """Small whole numbers and scales that are powers of two: every order of additions gives the same."""
    rng = np.random.default_rng(m + n)
    codes = rng.integers(-8, 8, size=(m, n)).astype(np.int8)
    scales = (2.0 ** rng.integers(-2, 3, size=(m, su.groups(n, 64)))).astype(np.float32)
    x = rng.integers(-15, 16, size=(batch, n)).astype(np.float64)
    y = call(biq, packed(biq, codes, scales, 64), su.to(x.astype(np.float32), kind), m, 64, "fp32")
    assert np.array_equal(su.back(y), x @ (codes * su.spread(scales.astype(np.float64), n, 64)).T)


@pytest.mark.parametrize("batch", [3, 20])
def test_magnitudes(biq, batch):
    """Vectors, and parts of a vector, of very different magnitudes."""
    codes, scales = weights(40, 1024, 128, 5)
    rng = np.random.default_rng(batch)
    x = rng.standard_normal((batch, 1024)) * np.repeat(10.0 ** rng.uniform(-8, 8, size=(batch, 8)), 128, axis=1)
    x[0] *= 1e25
    x[1] *= 1e-25
    x[2, 100:300] = 0
    t = su.to(x.astype(np.float32), "fp32")
    y = call(biq, packed(biq, codes, scales, 128), t, 40, 128, "fp32")
    for i in range(batch):
        check(y[i:i + 1], codes, scales, su.back(t)[i:i + 1], 128, "fp32")


@pytest.mark.parametrize("kind,batch", [("fp32", 5), ("bf16", 5), ("fp32", 40), ("fp16", 40)])
def test_infinities_and_nan_stay_in_their_vectors_and_rows(biq, kind, batch):
    codes, scales = weights(50, 600, 64, 5)
    codes[:, 7] = 3
    x = np.random.default_rng(1).standard_normal((batch, 600)).astype(np.float32)
    clean = call(biq, packed(biq, codes, scales, 64), su.to(x, kind), 50, 64, "fp32")
    x[1, 599], x[3, 7] = np.nan, np.inf
    scales[20, 2] = np.nan
    y = call(biq, packed(biq, codes, scales, 64), su.to(x, kind), 50, 64, "fp32")
    assert not torch.isfinite(y[1]).any() and not torch.isfinite(y[3]).any() and torch.isnan(y[:, 20]).all()
    vectors, cols = [i for i in range(batch) if i not in (1, 3)], [i for i in range(50) if i != 20]
    assert torch.equal(y[vectors][:, cols], clean[vectors][:, cols])


def test_strides_and_broadcast_inputs(biq):
    codes, scales = weights(40, 333, 32, 5)
    w = packed(biq, codes, scales, 32)
    for batch in (4, 30):
        x, _, values = inputs(1, 333, "bf16", 0, 7)
        y = call(biq, w, x.expand(batch, 333), 40, 32, "fp32")
        assert (y == y[0]).all()
        check(y[:1], codes, scales, values, 32, "fp32")
        big, _, values = inputs(batch, 999, "bf16", 0, 8)
        check(call(biq, w, big[:, 333:666], 40, 32, "fp32"), codes, scales, values[:, 333:666], 32, "fp32")


def test_same_result_twice(biq):
    codes, scales = weights(1000, 2048, 128, 5)
    w = packed(biq, codes, scales, 128)
    for batch in (1, 40):
        x, _, _ = inputs(batch, 2048, "fp32", 0, 9)
        assert torch.equal(call(biq, w, x, 1000, 128, "fp32"), call(biq, w, x, 1000, 128, "fp32"))
