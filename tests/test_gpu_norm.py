"""biq_norm against 64 bits; codes equal to the definition's in 32 bits."""
import numpy as np
import pytest
import torch

import step_util as su

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


def rows(count, n, typ, seed, big=1.0):
    """float32 arrays whose numbers the type holds."""
    rng = np.random.default_rng(seed)
    channel = np.exp(0.5 * rng.standard_normal(n))
    hold = lambda a: torch.from_numpy((a * big).astype(np.float32)).to(su.TYPES[typ]).float().numpy()
    return hold(rng.standard_normal((count, n)) * channel), hold(rng.standard_normal((count, n)) * channel * 3), \
        (1 + 0.3 * rng.standard_normal(n)).astype(np.float32)


def call(biq, x, residual, weight, typ, y_type=None, sums=False, codes=None, group=0, weight_add=0.0, eps=EPS, pad=0):
    """Outputs poisoned, rows `pad` elements further apart than they are long."""
    count, n = x.shape
    wide = lambda t: torch.full((count, n + pad), float("nan"), dtype=t, device="cuda:0")[:, :n]

    def strided(a):
        t = wide(su.TYPES[typ])
        t.copy_(torch.from_numpy(a))
        return t

    out = dict(y=wide(su.TYPES[y_type]) if y_type else None, sum=wide(su.TYPES[typ]) if sums else None, codes=None, scales=None)
    if codes:
        out["codes"] = torch.full((count, n + pad), 0x55, dtype=torch.uint8, device="cuda:0").view(torch.int8 if codes == "int8" else torch.float8_e4m3fn)[:, :n]
        out["scales"] = torch.full((count, su.groups(n, group)), float("nan"), device="cuda:0")
    biq.biq_norm(strided(x), weight=None if weight is None else torch.from_numpy(weight).to("cuda:0"),
                 residual=None if residual is None else strided(residual), group=group, weight_add=weight_add, eps=eps, **out)
    torch.cuda.synchronize()
    return out


def check(x, residual, weight, out, typ, y_type, weight_add=0.0, eps=EPS):
    """s is rounded once (2^-24 of it); the sum of squares has n terms, in 32 bits over at most 32 of them one after the other, then 10 levels of
    a tree: 2^-24 * 43 of it, half of that in r, with the division, the root, the mean and eps 4 more; two products."""
    s, r, y = su.norm(x.astype(np.float64), None if residual is None else residual.astype(np.float64),
                      None if weight is None else weight.astype(np.float64), weight_add, eps)
    w = (1 if weight is None else np.abs(weight)) + abs(weight_add)
    if out["sum"] is not None:
        got = su.back(out["sum"])
        assert (np.abs(got - s) <= su.HALF[typ] * np.abs(s) * (1 + 2.0 ** -12) + 2.0 ** -24 * np.abs(s) + 2.0 ** -25).all()
    if out["y"] is not None:
        got = su.back(out["y"])
        bound = 2.0 ** -24 * 30 * np.abs(s) * r * w + su.HALF[y_type] * np.abs(y) * (1 + 2.0 ** -12) + 2.0 ** -25
        assert (np.abs(got - y) <= bound).all(), np.max(np.abs(got - y) / bound)
    if out["codes"] is not None:
        fmt = "int8" if out["codes"].dtype == torch.int8 else "fp8"
        group = 0 if out["scales"].shape[1] == 1 and x.shape[1] > 128 else check.group
        codes, units = su.norm_codes(x, residual, weight, weight_add, group, fmt)
        assert np.array_equal(su.back(out["codes"].float()), codes)
        want = units.astype(np.float64) * r
        assert (np.abs(su.back(out["scales"]) - want) <= 2.0 ** -24 * 30 * want).all()


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("count,n", [(1, 1), (3, 2), (5, 7), (2, 8), (9, 63), (7, 512), (6, 513), (5, 2047), (3, 2049), (2, 4096), (3, 5003), (2, 8192),
                                     (2, 8193), (2, 16385), (2, 32768), (2, 32769), (1, 40001)])
def test_sizes(biq, typ, count, n):
    x, res, w = rows(count, n, typ, n)
    check(x, res, w, call(biq, x, res, w, typ, typ, True), typ, typ)
    check(x, None, None, call(biq, x, None, None, typ, "fp32"), typ, "fp32")


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("count,n", [(1, 1), (5, 31), (3, 33), (4, 300), (3, 1000), (2, 4097), (2, 9001), (2, 33000)])
def test_codes(biq, fmt, group, count, n):
    for typ, weight_add in (("bf16", 1.0), ("fp32", 0.0)):
        x, res, w = rows(count, n, typ, n + group)
        check.group = group
        out = call(biq, x, res, w - np.float32(weight_add), typ, "fp16", True, fmt, group, weight_add, pad=3)
        check(x, res, w - np.float32(weight_add), out, typ, "fp16", weight_add)


def test_types_of_the_output_and_strides(biq):
    x, res, w = rows(7, 777, "bf16", 3)
    for y_type in ("fp32", "bf16", "fp16"):
        for pad in (0, 1, 5, 8):
            check(x, res, w, call(biq, x, res, w, "bf16", y_type, True, pad=pad), "bf16", y_type)


@pytest.mark.parametrize("n", [300, 4096, 40000])
def test_in_place(biq, n):
    x, res, w = rows(5, n, "fp32", n)
    want = call(biq, x, res, w, "fp32", "fp32", True)
    tx, tr, tw = (su.to(a, "fp32") for a in (x, res, w))
    biq.biq_norm(tx, tx, weight=tw, residual=tr, sum=tr, eps=EPS)
    assert torch.equal(tx, want["y"]) and torch.equal(tr, want["sum"])
    tx = su.to(x, "fp32")
    biq.biq_norm(tx, tr, weight=tw, residual=su.to(res, "fp32"), sum=tx, eps=EPS)
    assert torch.equal(tr, want["y"]) and torch.equal(tx, want["sum"])


@pytest.mark.parametrize("n", [100, 3000, 40000])
def test_values_at_the_ends_of_the_range(biq, n):
    rng = np.random.default_rng(n)
    x = rng.standard_normal((6, n)).astype(np.float32)
    for i, by in enumerate((1e30, 1e-30, 0.0, 3e37, 1e-20, 1.0)):
        x[i] *= np.float32(by)
    check.group = 32
    for eps in (1e-6, 0.0):
        keep = x if eps else np.delete(x, 2, axis=0)                # (0 / 0 without eps)
        check(keep, None, None, call(biq, keep, None, None, "fp32", "fp32", codes="int8", group=32, eps=eps), "fp32", "fp32", eps=eps)


@pytest.mark.parametrize("n", [100, 3000, 40000])
def test_infinities_and_nan_stay_in_their_rows(biq, n):
    x = np.random.default_rng(n).standard_normal((5, n)).astype(np.float32)
    clean = call(biq, x, None, None, "fp32", "fp32", codes="int8", group=32)
    dirty = x.copy()
    dirty[1, n // 2], dirty[3, 0] = np.nan, np.inf
    out = call(biq, dirty, None, None, "fp32", "fp32", codes="int8", group=32)
    for i in (0, 2, 4):
        assert torch.equal(out["y"][i], clean["y"][i]) and torch.equal(out["codes"][i], clean["codes"][i]) and torch.equal(out["scales"][i], clean["scales"][i])
    assert torch.isnan(out["y"][1]).all() and torch.isnan(out["scales"][1]).all()
    assert torch.isnan(out["y"][3, 0]) and (out["y"][3, 1:] == 0).all()
    assert torch.isnan(out["scales"][3, 0]) and (out["scales"][3, 1:] == 0).all() and (out["codes"][3, :32] == 0).all()


def test_broadcast_rows_and_many_of_them(biq):
    x, _, w = rows(1, 96, "bf16", 8)
    y = torch.empty((70000, 96), dtype=torch.bfloat16, device="cuda:0")
    biq.biq_norm(su.to(x, "bf16").expand(70000, 96), y, weight=su.to(w, "fp32"), eps=EPS)
    assert (y == y[0]).all()
    check(x, None, w, dict(y=y[:1], sum=None, codes=None), "bf16", "bf16")
