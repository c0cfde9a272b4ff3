"""biq_attention_shared against softmax in 64 bits, and against biq_attention on the same pages."""
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
def held(shared, lens, heads, dim, page, fmt, seed=1):
    """Sequences of `lens` tokens whose first `shared` ones lie in the first one's pages."""
    pages = su.filled([max(lens[0], shared), *lens[1:]], heads, dim, page, fmt, seed)
    pages.lens[0] = lens[0]
    pages.table[1:, :shared // page] = pages.table[0, :shared // page]
    return pages


def call(biq, pages, q, shared, **how):
    """Output and lse of a call whose buffers are poisoned, and whose table has the shared pages for the first sequence only."""
    cache = pages.on(biq)
    cache.table[1:, :shared // pages.page] = -9
    ws = torch.full((biq.biq_attention_shared_workspace_bytes(cache, q, shared, **how),), 0xff, dtype=torch.uint8, device=q.device)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device=q.device)
    lse = torch.full(q.shape[:2], float("nan"), device=q.device)
    biq.biq_attention_shared(cache, q, out, shared, lse=lse, workspace=ws, **how)
    torch.cuda.synchronize()
    return out, lse


def check(biq, pages, shared, counts, q, typ, causal=True, window=0, scale=None, uniform=False, spare=0, **how):
    """spare: rows behind the last sequence's, which are left as they were.  Beside what biq_attention's sums over the tokens may cost there is an
    addition for every piece, of which there is one for every 4 steps at most and two more: counted as twice the steps."""
    scale = pages.dim ** -0.5 if scale is None else scale
    if not uniform:
        how.update(starts=au.starts_of(counts), max_rows=how.get("max_rows", max(counts)))
    out, lse = call(biq, pages, q.to("cuda:0"), shared, causal=causal, window=window, scale=scale, **how)
    out, lse = out.double().cpu(), lse.double().cpu()
    at = 0
    for s, n in enumerate(counts):
        length = int(pages.lens[s])
        m = min(n, how.get("max_rows", n))
        k, v = (torch.from_numpy(x) for x in pages.values(s))
        want, want_lse, size, vmax = au.softmax64(q[at:at + m].double(), k, v, scale, length - n + torch.arange(m), causal, window)
        tol, tol_lse = au.bounds(typ, want, size, vmax, 2 * length + 128)
        got, got_lse = out[at:at + m], lse[at:at + m]
        bad = ~((got - want).abs() <= tol)
        assert not bad.any(), (s, n, length, ((got - want).abs() / tol).max().item(), bad.sum().item(), bad.nonzero()[0].tolist())
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(got_lse), empty) and (got[empty] == 0).all()
        bad = ~((got_lse - want_lse).abs() <= tol_lse) & ~empty
        assert not bad.any(), (s, n, length, got_lse[bad][:3].tolist(), want_lse[bad][:3].tolist(), tol_lse)
        assert torch.isnan(out[at + m:at + n]).all() and torch.isnan(lse[at + m:at + n]).all()
        at += n
    assert torch.isnan(out[at:]).all() and torch.isnan(lse[at:]).all()
    return out, lse


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 128, 176, 192, 256])
def test_one_token_every_head_size(biq, fmt, typ, dim):
    pages = held(192, (193, 300, 192, 250), 2, dim, 32, fmt)
    check(biq, pages, 192, [1] * 4, au.rows_like([1] * 4, 6, dim, typ, dim), typ, uniform=True, max_len=300)


@pytest.mark.parametrize("shared", [16, 48, 64, 80, 256, 1040])
@pytest.mark.parametrize("page", [16, 48, 64, 256])
@pytest.mark.parametrize("own", [(1,), (1, 2), (15, 16, 17), (63, 64, 65, 66), (130, 1, 700)])
def test_lengths_and_pages(biq, shared, page, own):
    shared = -(-shared // page) * page
    pages = held(shared, tuple(shared + n for n in own), 2, 64, page, "int8")
    check(biq, pages, shared, [1] * len(own), au.rows_like([1] * len(own), 8, 64, "fp32", 3), "fp32", uniform=True)


@pytest.mark.parametrize("qh,heads", [(1, 1), (3, 3), (8, 1), (15, 3), (17, 1), (40, 2)])
@pytest.mark.parametrize("new", [1, 3, 5])
def test_shared_heads_and_drafted_tokens(biq, qh, heads, new):
    pages = held(128, (328, 218, 133, 129), heads, 64, 32, "fp8")
    check(biq, pages, 128, [new] * 4, au.rows_like([new] * 4, qh, 64, "fp32", qh), "fp32", uniform=True, max_len=328)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 37), (False, 0), (False, 50), (True, 200), (True, 1000)])
@pytest.mark.parametrize("dim", [64, 80, 128])
def test_prompts_ragged(biq, typ, causal, window, dim):
    """Prompts behind the prefix; one reaches into it, one has no rows in the call."""
    pages = held(144, (250, 400, 177, 229, 150), 2, dim, 48, "int8")
    counts = [106, 131, 1, 0, 140]
    check(biq, pages, 144, counts, au.rows_like(counts, 4, dim, typ, 9), typ, causal, window)


def test_large_heads_and_many_rows(biq):
    for dim, fmt, typ in ((256, "fp8", "bf16"), (192, "int8", "fp32")):
        pages = held(128, (400, 301), 1, dim, 64, fmt)
        check(biq, pages, 128, [270, 33], au.rows_like([270, 33], 3, dim, typ, 2), typ)


def test_many_sequences(biq):
    """More than a wave has lanes, some without rows."""
    rng = np.random.default_rng(4)
    lens = tuple(int(x) for x in 64 + rng.integers(1, 40, size=150))
    counts = [int(x) for x in rng.integers(0, 3, size=150)]
    pages = held(64, lens, 1, 64, 32, "int8")
    check(biq, pages, 64, counts, au.rows_like(counts, 2, 64, "fp32", 3), "fp32", max_len=104)
    check(biq, pages, 64, [1] * 150, au.rows_like([1] * 150, 2, 64, "bf16", 3), "bf16", uniform=True)


def test_sequences_shorter_than_the_prefix_and_rows_that_see_nothing(biq):
    pages = held(192, (100, 0, 192, 3, 260), 2, 64, 64, "int8")
    for counts in ([1] * 5, [5, 2, 4, 6, 3], [120, 1, 1, 1, 100]):
        for window in (0, 2, 70):
            check(biq, pages, 192, counts, au.rows_like(counts, 4, 64, "fp32", 1), "fp32", window=window)


def test_rows_of_no_sequence_and_beyond_max_rows_are_left(biq):
    pages = held(128, (200, 140, 180, 129), 2, 64, 32, "int8")
    counts = [37, 5, 20, 1]
    q = au.rows_like([*counts, 9], 4, 64, "bf16", 5)
    check(biq, pages, 128, counts, q, "bf16")
    for max_rows in (1, 7, 36):
        check(biq, pages, 128, counts, q, "bf16", max_rows=max_rows)
    # rows before the first sequence's
    q = q.to("cuda:0")
    want = call(biq, pages, q[:63], 128, starts=au.starts_of(counts), max_rows=37)
    got = call(biq, pages, torch.cat([q[63:], q[:63]]), 128, starts=au.starts_of(counts) + 9, max_rows=37)
    assert torch.isnan(got[0][:9]).all() and torch.allclose(got[0][9:].float(), want[0].float(), atol=0.02)


@pytest.mark.parametrize("max_len", [0, 1, 500, 900, 3000, 100000])
def test_the_split_does_not_depend_on_max_len_being_right(biq, max_len):
    pages = held(512, (3000, 600), 1, 64, 64, "int8")
    for counts, typ in (([1, 1], "fp32"), ([40, 40], "bf16")):
        check(biq, pages, 512, counts, au.rows_like(counts, 2, 64, typ, 4), typ, uniform=True, max_len=max_len)


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("scale", [0.0, -0.3, 12.0])
def test_scales(biq, new, scale):
    pages = held(320, (500, 390), 2, 64, 64, "int8")
    check(biq, pages, 320, [new] * 2, au.rows_like([new] * 2, 4, 64, "fp32", 6), "fp32", uniform=True, scale=scale)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_long_prefix(biq, dim, typ, fmt):
    """Pieces of many steps; few and many rows of all sequences."""
    pages = held(6016, (6017, 6100, 6500, 6079), 2, dim, 64, fmt)
    for new, qh in ((1, 4), (5, 8), (40, 8)):
        q = au.rows_like([new] * 4, qh, dim, typ, new)
        check(biq, pages, 6016, [new] * 4, q, typ, uniform=True, max_len=6500)
    check(biq, pages, 6016, [5] * 4, au.rows_like([5] * 4, 8, dim, typ, 1), typ, uniform=True, max_len=6500, window=3000)
    check(biq, pages, 6016, [40] * 4, au.rows_like([40] * 4, 8, dim, typ, 1), typ, uniform=True, max_len=6500, causal=False, window=444)


@pytest.mark.parametrize("dim,own", [(64, 1), (64, 300), (160, 70)])
def test_more_pieces_than_half_a_wave_has_lanes(biq, dim, own):
    """32 pieces of the prefix and an odd or even number of others."""
    pages = held(8192, (8192 + own, 8193), 1, dim, 256, "fp8")
    for window in (0, 40):
        check(biq, pages, 8192, [1, 1], au.rows_like([1, 1], 2, dim, "fp32", own), "fp32", uniform=True, max_len=8192 + own, window=window)


@pytest.mark.parametrize("new", [1, 130])
def test_what_is_hidden_does_not_show(biq, new):
    """NaN blocks outside a row's window and beyond a sequence's length; a page of the prefix that does not exist has no tokens."""
    pages = held(256, (420, 390), 2, 64, 32, "int8")
    q = au.rows_like([new] * 2, 4, 64, "fp32", 3).to("cuda:0")
    clean = call(biq, pages, q, 256, window=20 if new == 1 else 100)
    dirty = su.Pages.__new__(su.Pages)
    dirty.__dict__.update(pages.__dict__)
    dirty.store = pages.store.copy()
    for s in (0, 1):
        for b in range(0, (390 - new - 100) // 16 if new == 130 else 300 // 16):
            for h in (0, 1):
                for w in (0, 1):
                    _, _, at = dirty._where(s, b, h, w)
                    dirty.store[dirty.table[s, b * 16 // 32], at] = np.array([np.nan], np.float32).view(np.uint8)
    got = call(biq, dirty, q, 256, window=20 if new == 1 else 100)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    gone = su.Pages.__new__(su.Pages)
    gone.__dict__.update(pages.__dict__)
    gone.table = pages.table.copy()
    gone.table[:, 2] = 1 << 20
    out, _ = call(biq, gone, q, 256, causal=False)
    at = 0
    for s in (0, 1):
        k, v = (torch.from_numpy(x) for x in pages.values(s))
        keep = torch.ones(len(k), dtype=torch.bool)
        keep[64:96] = False
        want, _, size, vmax = au.softmax64(q[at:at + new].double().cpu(), k[keep], v[keep], 0.125, torch.zeros(new), False, 0)
        assert ((out[at:at + new].double().cpu() - want).abs() <= au.bounds("fp32", want, size, vmax, 1000)[0]).all()
        at += new


def test_strides_without_lse_and_the_same_result_twice(biq):
    pages = held(512, (700, 640, 513), 2, 64, 64, "int8")
    for new in (1, 60):
        q = au.rows_like([new] * 3, 4, 64, "bf16", 3).to("cuda:0")
        first, second = call(biq, pages, q, 512), call(biq, pages, q, 512)
        assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
        for pad in (1, 2, 4):
            wide = torch.full((3 * new, 5, 64 + pad), 9.0, dtype=torch.bfloat16, device="cuda:0")
            wide[:, :4, :64] = q
            out = torch.full_like(wide, 7.0)
            cache = pages.on(biq)
            ws = torch.empty(biq.biq_attention_shared_workspace_bytes(cache, wide[:, :4, :64], 512), dtype=torch.uint8, device="cuda:0")
            biq.biq_attention_shared(cache, wide[:, :4, :64], out[:, :4, :64], 512, workspace=ws)
            assert torch.equal(out[:, :4, :64], first[0]) and (out[:, 4] == 7).all() and (out[..., 64:] == 7).all()


def test_in_a_graph_while_lengths_grow(biq):
    """Lengths are device memory: a captured call serves the next tokens too."""
    pages = held(256, (260, 300, 257), 2, 64, 64, "int8")
    q = au.rows_like([1] * 3, 4, 64, "fp32", 3).to("cuda:0")
    cache = pages.on(biq)
    out = torch.empty_like(q)
    ws = torch.empty(biq.biq_attention_shared_workspace_bytes(cache, q, 256, max_len=320), dtype=torch.uint8, device="cuda:0")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        prepared = biq.PreparedSharedAttention(cache, q, out, 256, max_len=320, workspace=ws)
        prepared()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        prepared()
    for step in range(3):
        cache.lens.sub_(step)
        q.mul_(1.1)
        out.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(q)
        biq.biq_attention_shared(cache, q, want, 256, max_len=320, workspace=torch.empty_like(ws))
        assert torch.equal(out, want)
