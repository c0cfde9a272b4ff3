"""Calls whose grids have more than 2^32 threads go in several launches."""
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


def test_append_and_read(biq):
    """4096 sequences of 4 rows, 8 heads; max_rows left open stands for 16384 rows of each: 16.8 million workgroups."""
    seqs, heads, dim = 4096, 8, 16
    pages = torch.zeros((seqs, biq.biq_cache_page_bytes(16, heads, dim)), dtype=torch.uint8, device="cuda:0")
    table = torch.arange(seqs, dtype=torch.int32, device="cuda:0")[:, None].contiguous()
    lens = torch.full((seqs,), 9, dtype=torch.int32, device="cuda:0")
    k, v = (torch.randn((4 * seqs, heads, dim), device="cuda:0") for _ in range(2))
    starts = au.starts_of([4] * seqs)
    few, open_ = (biq.KvCache(pages.clone(), table, lens, 16, heads, dim) for _ in range(2))
    biq.biq_cache_append(few, k, v, starts=starts, max_rows=4)
    biq.biq_cache_append(open_, k, v, starts=starts)
    assert torch.equal(few.store, open_.store) and (few.store != pages).any(dim=1).all()
    a, b, c, d = (torch.full_like(k, 9.0) for _ in range(4))
    biq.biq_cache_read(few, a, b, starts=starts, max_rows=4)
    biq.biq_cache_read(few, c, d, starts=starts)
    assert torch.equal(a, c) and torch.equal(b, d) and (a != 9).all()


def test_attention(biq):
    """2048 sequences of 16 rows with max_rows left open: 8.4 million workgroups of 512."""
    seqs, heads, dim = 2048, 8, 16
    pages = su.filled([40], heads, dim, 64, "int8", 3)
    store = torch.from_numpy(pages.store[pages.table[0, :1]]).to("cuda:0")
    table = torch.zeros((seqs, 1), dtype=torch.int32, device="cuda:0")
    lens = (torch.arange(seqs, device="cuda:0") % 25 + 16).int()
    cache = biq.KvCache(store, table, lens, 64, heads, dim)
    q = torch.randn((16 * seqs, 4 * heads, dim), device="cuda:0")
    out, lse = au.call(biq, cache, q, starts=au.starts_of([16] * seqs))
    k, v = (torch.from_numpy(x) for x in pages.values(0))
    for s in (0, 1, 1000, 1023, 1024, 2046, 2047):
        length, rows = int(lens[s]), slice(16 * s, 16 * s + 16)
        want, want_lse, size, vmax = au.softmax64(q[rows].double().cpu(), k[:length], v[:length], dim ** -0.5, length - 16 + torch.arange(16), True, 0)
        tol, tol_lse = au.bounds("fp32", want, size, vmax, length)
        assert ((out[rows].double().cpu() - want).abs() <= tol).all(), s
        assert ((lse[rows].double().cpu() - want_lse).abs() <= tol_lse).all(), s
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_rotary(biq):
    """2^32 pairs and more, at odd addresses (a thread per pair): the first and the last rows are as in a small call."""
    heads, dim = 64, 128
    rows = (1 << 32) // (heads * dim // 2) + 33
    angles = torch.empty((64, dim // 2, 2), device="cuda:0")
    biq.biq_rotary_table(biq.biq_rotary_frequencies(dim).to("cuda:0"), angles)
    pos = (torch.arange(rows, device="cuda:0") % 64).int()
    wide = torch.empty((rows * heads * dim + 1,), dtype=torch.bfloat16, device="cuda:0")
    x = wide[1:].view(rows, heads, dim)
    x.copy_(torch.randn((1, heads, dim), device="cuda:0").bfloat16().expand(rows, heads, dim))
    some = torch.cat([torch.arange(70), torch.arange(rows // 2, rows // 2 + 70), torch.arange(rows - 70, rows)]).to("cuda:0")
    small = x[some].contiguous()
    want = torch.empty_like(small)
    biq.biq_rotary(small, want, pos[some].contiguous(), angles)
    biq.biq_rotary(x, x, pos, angles)
    assert torch.equal(x[some], want)
    first = x[:64].clone()
    for at in range(0, rows - 64, 65536):                       # every 64 rows are the same
        n = min(65536, (rows - at) // 64 * 64)
        assert (x[at:at + n].view(-1, 64, heads, dim) == first).all(), at


@pytest.mark.parametrize("drafts", [0, 2])
def test_verify(biq, drafts):
    """2^16 sequences of 2^20 tokens (the same rows for all of them): 2^24 workgroups for the sums."""
    seqs, vocab, dev = 1 << 16, 1 << 20, "cuda:0"
    z = torch.randn((drafts + 1, vocab), device=dev, generator=torch.Generator(device=dev).manual_seed(1))
    p = torch.softmax(z, dim=1)
    q = torch.softmax(z[:drafts] + 0.3, dim=1)
    t = torch.arange(seqs, dtype=torch.int32, device=dev)[:, None].repeat(1, drafts) % 1000
    u = (torch.arange(seqs, device=dev) % 1024 / 1024)[:, None].repeat(1, drafts + 1).contiguous()

    def run(s):
        n = s.numel()
        tokens, accepted = torch.empty((n, drafts + 1), dtype=torch.int32, device=dev), torch.empty(n, dtype=torch.int32, device=dev)
        ws = torch.empty(biq.biq_verify_workspace_bytes(n, vocab), dtype=torch.uint8, device=dev)
        biq.biq_verify_drafts(p.expand(n, -1, -1), q.expand(n, -1, -1) if drafts else None, t[s].contiguous(), u[s].contiguous(), tokens, accepted,
                              workspace=ws)
        return tokens, accepted

    tokens, accepted = run(torch.arange(seqs, device=dev))
    some = torch.cat([torch.arange(40), torch.arange(seqs // 2 - 20, seqs // 2 + 20), torch.arange(seqs - 40, seqs)]).to(dev)
    few, few_accepted = run(some)
    assert torch.equal(tokens[some], few) and torch.equal(accepted[some], few_accepted)
    assert (tokens.gather(1, accepted.long()[:, None]) >= 0).all()
