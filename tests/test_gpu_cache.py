"""The cache's writer and reader against their definition, code for code."""
import numpy as np
import pytest
import torch

import serving_util as su

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


def rows(counts, heads, dim, typ, seed, big=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((2, sum(counts), heads, dim), generator=g) * big
    return x[0].to(su.TYPES[typ]), x[1].to(su.TYPES[typ])


def starts_of(counts):
    return torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda:0")


def run_append(biq, pages, counts, k, v, uniform=False, **how):
    """Appends on the GPU and in numpy (lens grow by counts), compares every byte of the store."""
    pages.lens = (pages.lens + np.array(counts)).astype(np.int32)
    cache = pages.on(biq)
    if not uniform:
        how["starts"], how["max_rows"] = starts_of(counts), max(counts)
    biq.biq_cache_append(cache, k.to("cuda:0"), v.to("cuda:0"), **how)
    at = 0
    for s, n in enumerate(counts):
        pages.append(s, int(pages.lens[s]) - n, k[at:at + n].double().numpy(), v[at:at + n].double().numpy())
        at += n
    got = cache.store.cpu().numpy()
    assert np.array_equal(got, pages.store), np.argwhere(got != pages.store)[:5]
    return cache


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim", [16, 64, 80, 128, 192, 256])
def test_prompts_then_tokens(biq, fmt, typ, dim):
    """Ragged prompts, then tokens one by one through a block's end, growing so that older tokens are rounded anew; what lies
    beside the written blocks stays (the store starts as garbage)."""
    rng = np.random.default_rng(dim)
    pages = su.Pages([120, 90, 70, 60], 2, dim, 48, fmt, rng)
    pages.lens[:] = 0
    counts = [33, 1, 16, 0]
    run_append(biq, pages, counts, *rows(counts, 2, dim, typ, 1))
    for i in range(18):
        k, v = rows([1] * 4, 2, dim, typ, 2 + i, big=1.0 + 0.5 * i)
        run_append(biq, pages, [1] * 4, k, v, uniform=True)
    counts = [5, 40, 3, 20]
    run_append(biq, pages, counts, *rows(counts, 2, dim, typ, 50))


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (64, 32), (80, 80), (80, 2), (64, 22), (256, 64), (192, 190)])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_keys_are_turned_on_the_way(biq, fmt, interleaved, dim, rot, typ):
    """Products and sums of a pair rounded one by one, in the order of the definition."""
    rng = np.random.default_rng(dim)
    counts = [37, 3]
    pages = su.Pages([60, 30], 2, dim, 32, fmt, rng)
    pages.lens[:] = [20, 0]
    pages.append(0, 0, rng.standard_normal((20, 2, dim)), rng.standard_normal((20, 2, dim)))
    k, v = rows(counts, 2, dim, typ, 3)
    angles = torch.rand((64, rot // 2, 2), generator=torch.Generator().manual_seed(1)) * 2 - 1
    pos = torch.cat([torch.arange(20, 57), torch.arange(0, 3)])
    x, c, s = k.float(), angles[pos][:, None, :, 0], angles[pos][:, None, :, 1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    left, right = a * c - b * s, a * s + b * c
    y = x.clone()
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = left, right
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = left, right
    pages.lens = (pages.lens + np.array(counts)).astype(np.int32)
    cache = pages.on(biq)
    biq.biq_cache_append(cache, k.to("cuda:0"), v.to("cuda:0"), starts=starts_of(counts), angles=angles.to("cuda:0"), interleaved=interleaved)
    pages.append(0, 20, y[:37].double().numpy(), v[:37].double().numpy())
    pages.append(1, 0, y[37:].double().numpy(), v[37:].double().numpy())
    assert np.array_equal(cache.store.cpu().numpy(), pages.store)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_again_is_the_same_and_a_cut_back_sequence_goes_on(biq, fmt):
    rng = np.random.default_rng(1)
    pages = su.Pages([64], 1, 64, 32, fmt, rng)
    pages.lens[:] = 0
    k, v = rows([21], 1, 64, "fp32", 1)
    run_append(biq, pages, [21], k, v)
    k, v = rows([6], 1, 64, "fp32", 2, big=3.0)
    cache = run_append(biq, pages, [6], k, v)                   # tokens 21 .. 26
    before = cache.store.clone()
    biq.biq_cache_append(cache, k.to("cuda:0"), v.to("cuda:0"))
    assert torch.equal(before, cache.store)
    pages.lens[:] = 23                                          # 4 drafted tokens refused
    k, v = rows([2], 1, 64, "fp32", 3, big=0.1)
    run_append(biq, pages, [2], k, v)                           # ... the block keeps the scale, later tokens are zeros
    pages.lens[:] = 16
    k, v = rows([1], 1, 64, "fp32", 4, big=0.1)
    run_append(biq, pages, [1], k, v)                           # its first token written again: a scale of its own


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_zeros_tiny_huge_and_no_numbers(biq, fmt):
    rng = np.random.default_rng(1)
    top = {"int8": 127.0, "fp8": 448.0}[fmt]
    x = torch.zeros((112, 1, 64))
    x[0:16] = 0.0
    x[16:32] = 2.0 ** -101                                      # held as zeros
    x[32:48] = torch.randn((16, 1, 64)) * 2.0 ** -90
    x[48:64] = torch.randn((16, 1, 64)) * 1e37
    x[64:80, :, ::2] = top                                      # codes on the edge, ties
    x[64:80, :, 1::2] = torch.arange(32.0)[None, None, :] + 0.5
    x[80:96] = 1.0
    x[85, 0, 3] = float("nan")
    x[96:112] = 1.0
    x[100, 0, 9] = float("-inf")
    pages = su.Pages([120], 1, 64, 16, fmt, rng)
    pages.lens[:] = 0
    run_append(biq, pages, [112], x, x.flip(0).contiguous())
    pages.lens[:] = 85                                          # the NaN's block goes on being NaN
    k, v = rows([3], 1, 64, "fp32", 3)
    run_append(biq, pages, [3], k, v)
    pages.lens[:] = 80
    run_append(biq, pages, [3], k, v)                           # written from its first token on: numbers again
    assert np.isfinite(pages.block(0, 5, 0, 0)[1])


def test_positions_without_angles_and_pages_that_do_not_exist(biq):
    rng = np.random.default_rng(1)
    pages = su.Pages([64], 1, 64, 16, "int8", rng)
    pages.lens[:] = 40
    cache = pages.on(biq)
    angles = torch.ones((20, 32, 2), device="cuda:0")           # tokens 20 .. have none
    k, v = rows([40], 1, 64, "fp32", 3)
    biq.biq_cache_append(cache, k.to("cuda:0"), v.to("cuda:0"), angles=angles)
    out = torch.zeros((40, 1, 64), device="cuda:0")
    values = torch.zeros_like(out)
    biq.biq_cache_read(cache, out, values)
    assert torch.isfinite(out[:16]).all() and torch.isnan(out[16:]).all() and torch.isfinite(values).all()
    for bad in (-1, pages.store.shape[0], 1 << 30):
        pages = su.Pages([64], 1, 64, 16, "int8", rng)
        pages.lens[:] = 40
        page = pages.table[0, 1]
        pages.table[0, 1] = bad
        cache = pages.on(biq)
        biq.biq_cache_append(cache, k.to("cuda:0"), v.to("cuda:0"))
        changed = (cache.store.cpu().numpy() != pages.store).any(axis=1)
        assert changed[pages.table[0, 0]] and changed[pages.table[0, 2]] and changed.sum() == 2 and not changed[page]
        out.fill_(5.0)
        biq.biq_cache_read(cache, out, values)
        assert (out[16:32] == 0).all() and (out[:16] != 0).any() and (out[32:] != 0).any()


def test_more_rows_than_tokens(biq):
    """Rows before token 0 are dropped, and read as zeros."""
    rng = np.random.default_rng(1)
    pages = su.Pages([64, 64], 2, 64, 16, "int8", rng)
    pages.lens[:] = [7, 0]
    k, v = rows([20, 20], 2, 64, "fp32", 3)
    cache = pages.on(biq)
    biq.biq_cache_append(cache, k.to("cuda:0"), v.to("cuda:0"))
    pages.append(0, 0, k[13:20].double().numpy(), v[13:20].double().numpy())
    assert np.array_equal(cache.store.cpu().numpy(), pages.store)
    a, b = (torch.full((40, 2, 64), 9.0, device="cuda:0") for _ in range(2))
    biq.biq_cache_read(cache, a, b)
    want = pages.values(0)
    assert (a[:13] == 0).all() and (a[20:] == 0).all() and np.array_equal(a[13:20].cpu().numpy(), want[0].astype(np.float32))
    assert (b[:13] == 0).all() and (b[20:] == 0).all() and np.array_equal(b[13:20].cpu().numpy(), want[1].astype(np.float32))


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim", [16, 80, 128, 256])
def test_read(biq, fmt, typ, dim):
    pages = su.filled([100, 33, 7], 2, dim, 48, fmt, 2)
    counts = [100, 20, 10]
    a, b = (torch.full((sum(counts) + 2, 3, dim + 3), 9.0, dtype=su.TYPES[typ], device="cuda:0") for _ in range(2))
    biq.biq_cache_read(pages.on(biq), a[:130, 1:, :dim], b[:130, :2, 1:dim + 1], starts=starts_of(counts))
    at = 0
    for s, n in enumerate(counts):
        for got, want in zip((a[at:at + n, 1:, :dim], b[at:at + n, :2, 1:dim + 1]), pages.values(s)):
            full = np.zeros((n, 2, dim), np.float32)
            have = min(n, int(pages.lens[s]))
            full[n - have:] = want[len(want) - have:]
            assert torch.equal(got.cpu(), torch.from_numpy(full).to(su.TYPES[typ]))
        at += n
    assert (a[130:] == 9).all() and (a[:, 0] == 9).all() and (a[..., dim:] == 9).all()
    assert (b[130:] == 9).all() and (b[:, 2] == 9).all() and (b[..., 0] == 9).all()


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_strides_of_the_rows(biq, typ):
    """Keys and values as parts of a projection's rows, at odd addresses."""
    rng = np.random.default_rng(1)
    wide = torch.randn((23 * 7 * 64 + 1,), generator=torch.Generator().manual_seed(1)).to(su.TYPES[typ])
    for lead in (0, 1):
        x = wide[lead:lead + 23 * 7 * 64].view(23, 7, 64)
        pages = su.Pages([64], 2, 64, 32, "int8", rng)
        pages.lens[:] = 23
        cache = pages.on(biq)
        gpu = wide.to("cuda:0")[lead:lead + 23 * 7 * 64].view(23, 7, 64)
        biq.biq_cache_append(cache, gpu[:, 3:5], gpu[:, 5:7])
        pages.append(0, 0, x[:, 3:5].double().numpy(), x[:, 5:7].double().numpy())
        assert np.array_equal(cache.store.cpu().numpy(), pages.store)
