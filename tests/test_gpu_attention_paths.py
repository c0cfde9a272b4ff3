"""biq_attention on each of its kernels: tokens shared by workgroups and joined, and many rows, for every size of head."""
import functools

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


@functools.lru_cache(maxsize=4)
def held(lens, heads, dim, page, fmt, seed):
    return su.filled(list(lens), heads, dim, page, fmt, seed)


# ---- few rows: the workgroups share all steps, what they have of a unit is joined -------------------------------

@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 80, 96, 128, 160, 192, 256])
def test_shared_steps_every_head_size(biq, dim, typ, fmt):
    """One token, and five whose rows with their heads take two tiles; lengths from 0 to 40 steps."""
    lens = (2500, 700, 64, 1100, 0, 63)
    pages = held(lens, 2, dim, 48, fmt, dim)
    for new, qh, window in ((1, 8, 0), (1, 6, 900), (5, 8, 0)):
        q = au.rows_like([new] * 6, qh, dim, typ, dim + new)
        assert biq.biq_attention_workspace_bytes(pages.on(biq), q.to("cuda:0"), max_len=2500) > 0      # (it is shared and joined)
        au.check(biq, pages, [new] * 6, q, typ, window=window, max_len=2500)


@pytest.mark.parametrize("dim", [128, 256])
def test_shared_steps_negative_scale_not_causal_and_again(biq, dim):
    pages = held((2500, 700, 64, 1100, 0, 63), 2, dim, 48, "int8", dim)
    q = au.rows_like([5] * 6, 8, dim, "bf16", 7)
    for how in (dict(causal=False, window=0), dict(causal=False, window=70), dict(scale=-0.05)):
        first = au.check(biq, pages, [5] * 6, q, "bf16", max_len=2500, **how)
        again = au.check(biq, pages, [5] * 6, q, "bf16", max_len=2500, **how)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ---- many rows --------------------------------------------------------------------------------------------------

LENS, COUNTS, HEADS, QH = (150, 70, 400, 33), [150, 70, 200, 0], 16, 96


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
def test_many_rows_whole_heads(biq, dim, typ, fmt):
    pages = held(LENS, HEADS, dim, 48, fmt, dim)
    q = au.rows_like(COUNTS, QH, dim, typ, dim)
    au.check(biq, pages, COUNTS, q, typ)
    au.check(biq, pages, COUNTS, q, typ, window=90, sample=range(0, 200, 7))


@pytest.mark.parametrize("dim", [16, 32, 48, 144, 160, 176, 208, 224])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_many_rows_heads_between_multiples_of_64(biq, typ, dim):
    pages = held(LENS, HEADS, dim, 64, "int8", dim)
    au.check(biq, pages, COUNTS, au.rows_like(COUNTS, QH, dim, typ, dim), typ, window=90)


@pytest.mark.parametrize("dim", [32, 80, 128, 192])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_many_rows_not_causal_windows_scales_and_again(biq, typ, dim):
    pages = held(LENS, HEADS, dim, 48, "fp8", dim)
    q = au.rows_like(COUNTS, QH, dim, typ, dim)
    for how in (dict(causal=False), dict(causal=False, window=50), dict(window=1), dict(scale=-0.05), dict(scale=0.0), dict(scale=3.0)):
        first = au.check(biq, pages, COUNTS, q, typ, sample=range(0, 200, 9), **how)
    again = au.check(biq, pages, COUNTS, q, typ, sample=range(0, 200, 9), **how)
    assert torch.equal(first[0].nan_to_num(), again[0].nan_to_num()) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_many_rows_before_the_first_token(biq, typ, dim):
    counts = [200, 150, 60, 40]                                 # of 150, 70, 400 and 33 tokens
    pages = held(LENS, HEADS, dim, 48, "int8", dim)
    q = au.rows_like(counts, QH, dim, typ, 5)
    for window in (0, 20):
        _, lse = au.check(biq, pages, counts, q, typ, window=window, sample=range(0, 200, 3))
        assert torch.isinf(lse[:50]).all() and torch.isinf(lse[200:280]).all()
    au.check(biq, pages, counts, q, typ, causal=False, window=20, sample=range(0, 200, 3))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_many_rows_what_is_hidden_does_not_show(biq, typ, dim):
    """A NaN block outside most rows' windows, a page that does not exist, no page at all."""
    pages = su.filled([400], HEADS, dim, 32, "fp8", dim)
    for h in range(HEADS):
        for w in (0, 1):
            pages.put(0, 1, h, w, np.zeros((16, dim)), np.float32("nan"))       # tokens 16 .. 31
    q = au.rows_like([300], QH, dim, typ, 1).to("cuda:0")
    how = dict(causal=True, max_len=400)
    out, lse = au.call(biq, pages.on(biq), q, window=60, **how)                 # rows see tokens from 41 + row on
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    out, lse = au.call(biq, pages.on(biq), q, window=100, **how)                # from 1 + row on: the first 31 rows see the block
    seen = torch.arange(300, device="cuda:0") <= 30
    assert torch.isnan(out[seen]).all() and torch.isfinite(out[~seen]).all() and torch.isfinite(lse[~seen]).all()
    k, v = (torch.from_numpy(x) for x in pages.values(0))
    pages.table[0, 0] = 1 << 30                                 # tokens 0 .. 31 gone
    out, lse = au.call(biq, pages.on(biq), q, **how)
    pick = torch.arange(0, 300, 23)
    want, want_lse, size, vmax = au.softmax64(q[pick].double().cpu(), k[32:], v[32:], dim ** -0.5, 100 + pick - 32, True, 0)
    tol, tol_lse = au.bounds(typ, want, size, vmax, 400)
    assert ((out[pick].double().cpu() - want).abs() <= tol).all() and ((lse[pick].double().cpu() - want_lse).abs() <= tol_lse).all()
    pages.table[:] = -1
    out, lse = au.call(biq, pages.on(biq), q, **how)
    assert (out == 0).all() and torch.isinf(lse).all()


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_many_rows_a_nan_stays_in_its_row_and_head(biq, typ):
    pages = held(LENS, HEADS, 64, 48, "int8", 64)
    q = au.rows_like(COUNTS, QH, 64, typ, 1)
    how = dict(starts=au.starts_of(COUNTS), max_rows=200)
    want, want_lse = au.call(biq, pages.on(biq), q.to("cuda:0"), **how)
    hit = torch.zeros((sum(COUNTS), QH), dtype=torch.bool, device="cuda:0")
    for row, head, value in ((3, 1, float("nan")), (149, 95, float("inf")), (151, 0, float("-inf")), (300, 50, float("nan"))):
        q[row, head, 5] = value
        hit[row, head] = True
    got, lse = au.call(biq, pages.on(biq), q.to("cuda:0"), **how)
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 80])
def test_many_rows_strides_and_alignment(biq, typ, dim):
    pages = held(LENS, HEADS, dim, 48, "int8", dim)
    rows, how = sum(COUNTS), dict(starts=au.starts_of(COUNTS), max_rows=200)
    q = au.rows_like(COUNTS, QH, dim, typ, 1).to("cuda:0")
    cache = pages.on(biq)
    want, _ = au.call(biq, cache, q, **how)
    ws = torch.empty(max(16, biq.biq_attention_workspace_bytes(cache, q, **how)), dtype=torch.uint8, device="cuda:0")
    for lead, heads, width in ((1, QH + 1, dim), (0, QH, dim + 3), (2, QH + 2, dim + 16)):
        size = rows * heads * width
        wide = torch.full((size + 8,), float("nan"), dtype=q.dtype, device="cuda:0")
        view = wide[lead:lead + size].view(rows, heads, width)[:, heads - QH:, :dim]
        view.copy_(q)
        dest = torch.full_like(wide, 7.0)
        out = dest[lead:lead + size].view(rows, heads, width)[:, heads - QH:, :dim]
        biq.biq_attention(cache, view, out, workspace=ws, **how)
        assert torch.equal(out, want)
        out.fill_(7.0)
        assert (dest == 7.0).all()                              # nothing beside the heads was written
    turned = q.transpose(0, 1).contiguous().transpose(0, 1)     # heads outermost
    out = torch.empty_like(q)
    biq.biq_attention(cache, turned, out, workspace=ws, **how)
    assert torch.equal(out, want)


def test_many_rows_in_a_graph(biq):
    pages = held(LENS, HEADS, 128, 48, "int8", 128)
    cache, how = pages.on(biq), dict(starts=au.starts_of(COUNTS), max_rows=200)
    q = au.rows_like(COUNTS, QH, 128, "bf16", 1).to("cuda:0")
    out = torch.zeros_like(q)
    au.call(biq, cache, q, **how)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        biq.biq_attention(cache, q, out, **how)
    for _ in range(3):
        q.copy_(torch.randn_like(q))
        want, _ = au.call(biq, cache, q, **how)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("dim", [16, 32, 48])
@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
def test_many_rows_that_fill_the_gpu_small_heads(biq, typ, dim):
    """Rows enough for workgroups of eight waves; a sample of them is checked."""
    lens, counts = (1100, 700, 1500), [1100, 650, 1300]
    pages = held(lens, 16, dim, 64, "int8", dim)
    q = au.rows_like(counts, 96, dim, typ, 3)
    for window in (0, 200):
        au.check(biq, pages, counts, q, typ, window=window, sample=[0, 1, 217, 649, 1057, 1299])
