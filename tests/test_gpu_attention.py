"""biq_attention against softmax in 64 bits on the same codes."""
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


def call(biq, cache, q, **how):
    """Output and lse of a call whose buffers are poisoned."""
    ws = torch.full((max(16, biq.biq_attention_workspace_bytes(cache, q, **how)),), 0xff, dtype=torch.uint8, device=q.device)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device=q.device)
    lse = torch.full(q.shape[:2], float("nan"), device=q.device)
    biq.biq_attention(cache, q, out, lse=lse, workspace=ws, **how)
    torch.cuda.synchronize()
    return out, lse


def check(biq, pages, counts, typ, qh, seed, causal=True, window=0, uniform=False, scale=None, max_len=0):
    rng = np.random.default_rng(seed)
    rows, dim = sum(counts), pages.dim
    q = torch.from_numpy(rng.standard_normal((rows, qh, dim)).astype(np.float32) * 1.5).to(su.TYPES[typ])
    how = dict(causal=causal, window=window, max_len=max_len)
    if scale is not None:
        how["scale"] = scale
    if not uniform:
        how["starts"] = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda:0")
        how["max_rows"] = max(counts)
    out, lse = call(biq, pages.on(biq), q.to("cuda:0"), **how)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    at = 0
    for s, n in enumerate(counts):
        length = int(pages.lens[s])
        k, v = pages.values(s)
        want, want_lse, size, vmax = su.attention(q[at:at + n].double().numpy(), k, v, dim ** -0.5 if scale is None else scale,
                                                  np.arange(length - n, length), causal, window)
        tol, tol_lse = su.attention_bounds(typ, want, size, vmax)
        err = np.abs(out[at:at + n] - want)
        assert np.all(err <= tol), (s, n, length, np.nanmax(err / tol), np.isnan(err).sum())
        empty = np.isinf(want_lse)
        assert np.array_equal(np.isinf(lse[at:at + n]), empty) and np.all(out[at:at + n][empty] == 0)
        assert np.all(np.abs(lse[at:at + n][~empty] - want_lse[~empty]) <= tol_lse), s
        at += n


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 128, 176, 192, 256])
def test_one_token_every_head_size(biq, fmt, typ, dim):
    check(biq, su.filled([1, 15, 64, 129], 2, dim, 32, fmt, dim), [1, 1, 1, 1], typ, 6, dim, uniform=True)


@pytest.mark.parametrize("lens", [[1], [2], [16], [17], [63, 64, 65], [127, 128, 129, 130], [511, 513, 700], [1500, 3, 0]])
@pytest.mark.parametrize("page", [16, 48, 64, 112, 256])
def test_lengths_and_pages(biq, lens, page):
    check(biq, su.filled(lens, 2, 64, page, "int8", len(lens) + page), [1] * len(lens), "fp32", 8, 3, uniform=True)


@pytest.mark.parametrize("qh,heads", [(1, 1), (3, 3), (8, 1), (15, 3), (16, 1), (17, 1), (40, 2), (64, 1)])
@pytest.mark.parametrize("new", [1, 3, 5])
def test_shared_heads_and_drafted_tokens(biq, qh, heads, new):
    check(biq, su.filled([200, 90, 5], heads, 64, 32, "fp8", qh), [new] * 3, "fp32", qh, qh, uniform=True)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 37), (False, 0), (False, 50), (True, 1000)])
@pytest.mark.parametrize("dim", [64, 80, 128])
def test_prompts_ragged(biq, typ, causal, window, dim):
    """Prompts of several sizes, over what a sequence had before; one sequence has no rows in the call."""
    check(biq, su.filled([150, 300, 33, 129, 70], 2, dim, 48, "int8", 5), [150, 131, 1, 0, 70], typ, 4, 9, causal, window)


def test_prompt_of_many_rows_and_large_heads(biq):
    check(biq, su.filled([400], 1, 256, 64, "fp8", 1), [333], "bf16", 3, 2)
    check(biq, su.filled([400], 1, 192, 64, "int8", 1), [290], "fp32", 2, 2)


def test_rows_before_the_first_token_see_nothing(biq):
    """More rows than tokens: the first rows lie before token 0."""
    check(biq, su.filled([3, 0, 40], 2, 64, 16, "int8", 1), [5, 2, 60], "fp32", 4, 1)
    check(biq, su.filled([3, 0, 40], 2, 64, 16, "fp8", 1), [5, 2, 60], "bf16", 4, 1, causal=True, window=2)


def test_the_split_does_not_depend_on_max_len_being_right(biq):
    pages = su.filled([3000], 1, 64, 64, "int8", 4)
    for max_len in (0, 1, 64, 700, 3000, 100000):
        check(biq, pages, [1], "fp32", 2, 4, uniform=True, max_len=max_len)
        check(biq, pages, [40], "bf16", 2, 4, uniform=True, max_len=max_len)


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("scale", [0.0, -0.3, 12.0])
def test_scales(biq, new, scale):
    check(biq, su.filled([500], 2, 64, 64, "int8", 6), [new], "fp32", 4, 6, uniform=True, scale=scale)


@pytest.mark.parametrize("new", [1, 130])
def test_what_is_hidden_does_not_show(biq, new):
    """NaN blocks and codes outside a row's window, beyond its length and on missing pages; a page that does not exist has no
    tokens."""
    pages = su.filled([400], 2, 64, 32, "fp8", 8)
    nan = np.float32("nan")
    for h in range(2):
        for w in (0, 1):
            pages.put(0, 1, h, w, np.zeros((16, 64)), nan)      # tokens 16 .. 31
    q = torch.randn((new, 4, 64), generator=torch.Generator().manual_seed(1)).to("cuda:0")
    out, lse = call(biq, pages.on(biq), q, causal=True, window=100)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    out, _ = call(biq, pages.on(biq), q, causal=True)
    assert torch.isnan(out).all()                               # all rows see the block
    k, v = pages.values(0)
    pages.table[0, 0] = 1 << 30                                 # tokens 0 .. 31 gone
    out, lse = call(biq, pages.on(biq), q, causal=True)
    for r in range(0, new, 43):
        want, want_lse, size, vmax = su.attention(q[r:r + 1].double().cpu().numpy(), k[32:], v[32:], 0.125, np.array([400 - new + r - 32]), True, 0)
        tol, tol_lse = su.attention_bounds("fp32", want, size, vmax)
        assert np.all(np.abs(out[r:r + 1].double().cpu().numpy() - want) <= tol)
        assert np.all(np.abs(lse[r:r + 1].double().cpu().numpy() - want_lse) <= tol_lse)
    pages.table[:] = -1
    out, lse = call(biq, pages.on(biq), q, causal=True)
    assert (out == 0).all() and torch.isinf(lse).all()


def test_a_nan_stays_in_its_row_and_head(biq):
    pages = su.filled([300, 300], 2, 64, 32, "int8", 8)
    for new in (1, 70):
        q = torch.randn((2 * new, 4, 64), generator=torch.Generator().manual_seed(1))
        want, _ = call(biq, pages.on(biq), q.to("cuda:0"))
        q[new - 1, 1, 5] = float("nan")
        q[new, 2, 7] = float("inf")
        got, lse = call(biq, pages.on(biq), q.to("cuda:0"))
        hit = torch.zeros((2 * new, 4), dtype=torch.bool, device="cuda:0")
        hit[new - 1, 1] = hit[new, 2] = True
        assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("new", [1, 70])
def test_strides_and_alignment(biq, typ, new):
    pages = su.filled([200, 77], 2, 80, 32, "int8", 8)
    q = torch.randn((2 * new, 4, 80), generator=torch.Generator().manual_seed(1)).to(su.TYPES[typ]).to("cuda:0")
    want, _ = call(biq, pages.on(biq), q)
    for lead, heads, width in ((1, 5, 80), (0, 4, 83), (2, 6, 96)):
        wide = torch.full((2 * new * heads * width + 8,), float("nan"), dtype=q.dtype, device="cuda:0")
        view = wide[lead:lead + 2 * new * heads * width].view(2 * new, heads, width)[:, 1 if heads > 4 else 0:, :80][:, :4]
        view.copy_(q)
        dest = torch.full_like(wide, 7.0)
        out = dest[lead:lead + 2 * new * heads * width].view(2 * new, heads, width)[:, 1 if heads > 4 else 0:, :80][:, :4]
        cache = pages.on(biq)
        ws = torch.empty(max(16, biq.biq_attention_workspace_bytes(cache, view)), dtype=torch.uint8, device="cuda:0")
        biq.biq_attention(cache, view, out, workspace=ws)
        assert torch.equal(out, want)
        out.fill_(7.0)
        assert (dest == 7.0).all()                              # nothing beside the heads was written
    turned = q.transpose(0, 1).contiguous().transpose(0, 1)     # heads outermost
    out = torch.empty_like(q)
    ws = torch.empty(max(16, biq.biq_attention_workspace_bytes(cache, turned)), dtype=torch.uint8, device="cuda:0")
    biq.biq_attention(cache, turned, out, workspace=ws)
    assert torch.equal(out, want)


def test_another_stream_and_a_graph(biq):
    pages = su.filled([900, 20], 2, 64, 64, "int8", 8)
    cache = pages.on(biq)
    q = torch.randn((2, 8, 64), device="cuda:0")
    want, _ = call(biq, cache, q, max_len=900)
    out = torch.zeros_like(q)
    ws = torch.empty(max(16, biq.biq_attention_workspace_bytes(cache, q, max_len=900)), dtype=torch.uint8, device="cuda:0")
    assert ws.numel() > 16                                      # (a call that is split and joined)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    biq.biq_attention(cache, q, out, max_len=900, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        biq.biq_attention(cache, q, out, max_len=900, workspace=ws)
    for _ in range(3):
        q.copy_(torch.randn_like(q))
        want, _ = call(biq, cache, q, max_len=900)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_the_same_bits_every_time(biq):
    cache = su.filled([2000], 2, 64, 64, "fp8", 8).on(biq)
    for new in (1, 200):
        q = torch.randn((new, 8, 64), device="cuda:0")
        first, _ = call(biq, cache, q)
        for _ in range(3):
            assert torch.equal(first, call(biq, cache, q)[0])


def test_parts_join_by_their_lse(biq):
    """A context in two calls, joined by what lse says."""
    pages = su.filled([500], 2, 64, 32, "int8", 8)
    q = torch.randn((1, 4, 64), device="cuda:0")
    want, want_lse = call(biq, pages.on(biq), q, causal=False)
    a, la = call(biq, pages.on(biq, lens=[320]), q, causal=False)
    pages.table[0, :6] = pages.table[0, 10:16]
    b, lb = call(biq, pages.on(biq, lens=[180]), q, causal=False)
    lse = torch.logaddexp(la, lb)
    joined = a * (la - lse).exp()[..., None] + b * (lb - lse).exp()[..., None]
    assert (joined - want).abs().max() < 1e-5 and (lse - want_lse).abs().max() < 1e-5


def test_offsets_beyond_32_bits(biq):
    """Pages that lie above 4 GiB of the store."""
    page, heads, dim = 256, 8, 256
    size = biq.biq_cache_page_bytes(page, heads, dim)
    count = (1 << 32) // size + 40
    pages = su.filled([700], heads, dim, page, "int8", 3)
    store = torch.zeros((count, size), dtype=torch.uint8, device="cuda:0")
    table = torch.tensor([[count - 1, count - 30, count - 7]], dtype=torch.int32, device="cuda:0")
    for i in range(3):
        store[table[0, i]] = torch.from_numpy(pages.store[pages.table[0, i]]).to("cuda:0")
    q = torch.randn((1, 16, dim), device="cuda:0")
    want, _ = call(biq, pages.on(biq), q)
    lens = torch.tensor([700], dtype=torch.int32, device="cuda:0")
    cache = biq.KvCache(store, table, lens, page, heads, dim, "int8")
    for rows in (1, 40):
        q = torch.randn((rows, 16, dim), device="cuda:0")
        assert torch.equal(call(biq, cache, q, max_len=1024)[0], call(biq, pages.on(biq), q, max_len=1024)[0])


@pytest.mark.parametrize("seqs,new", [(70, 1), (130, 1), (66, 9)])
def test_many_sequences_share_the_work(biq, seqs, new):
    """More sequences than lanes, lengths from none to many: places, pieces and their joining."""
    rng = np.random.default_rng(seqs)
    lens = [int(n) for n in rng.choice([0, 1, 30, 64, 65, 200, 640, 1500], size=seqs)]
    counts = [0 if s % 11 == 5 else int(rng.integers(1, new + 1)) for s in range(seqs)]
    check(biq, su.filled(lens, 1, 32, 64, "int8", seqs), counts, "fp32", 2, seqs, max_len=1500)


def test_one_long_sequence_is_shared(biq):
    check(biq, su.filled([9000], 1, 32, 256, "int8", 1), [1], "fp32", 3, 1, uniform=True)
    check(biq, su.filled([9000, 0, 17], 1, 32, 256, "fp8", 1), [6, 1, 2], "bf16", 3, 1, window=5000)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [32, 80, 96, 112, 160, 224])
def test_prompts_heads_between_multiples_of_64(biq, fmt, typ, dim):
    """Rows enough for the kernel of many rows, whatever the size of the head."""
    check(biq, su.filled([150, 70, 400], 16, dim, 48, fmt, dim), [150, 70, 200], typ, 64, dim, True, 90)


@pytest.mark.parametrize("dim,typ,window", [(64, "bf16", 0), (80, "fp32", 300), (128, "fp16", 0)])
def test_prompts_that_fill_the_gpu(biq, dim, typ, window):
    """Rows enough for the widest workgroups (ragged, the last of them partly filled); a sample of them is checked."""
    lens, counts = [1100, 700, 1500], [1100, 650, 1300]
    heads, qh = 16, 96
    pages = su.filled(lens, heads, dim, 64, "int8", dim)
    rng = np.random.default_rng(1)
    q = torch.from_numpy(rng.standard_normal((sum(counts), qh, dim)).astype(np.float32)).to(su.TYPES[typ])
    starts = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda:0")
    out, lse = call(biq, pages.on(biq), q.to("cuda:0"), starts=starts, max_rows=max(counts), max_len=1500, window=window)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    at = 0
    for s, n in enumerate(counts):
        k, v = pages.values(s)
        for r in sorted({0, 1, n // 3, n - 43, n - 1}):
            for h in (0, 5, 47, 95):
                g = h // 6
                want, want_lse, size, vmax = su.attention(q[at + r:at + r + 1, h:h + 1].double().numpy(), k[:, g:g + 1], v[:, g:g + 1], dim ** -0.5,
                                                          np.array([lens[s] - n + r]), True, window)
                tol, tol_lse = su.attention_bounds(typ, want, size, vmax)
                assert np.all(np.abs(out[at + r, h] - want[0, 0]) <= tol[0, 0]), (s, r, h)
                assert abs(lse[at + r, h] - want_lse[0, 0]) <= tol_lse, (s, r, h)
        at += n


@pytest.mark.parametrize("new", [1, 100])
def test_a_window_as_large_as_can_be(biq, new):
    pages = su.filled([300, 50], 1, 64, 64, "int8", 3)
    for window in (299, 300, 301, 384, 385, 2**31 - 1):
        check(biq, pages, [new, 70], "fp32", 2, 5, window=window)
