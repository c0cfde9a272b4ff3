"""Ragged calls at their bounds: sequences with more rows than max_rows."""
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


@functools.lru_cache(maxsize=None)
def held(lens, heads, dim):
    return su.filled(list(lens), heads, dim, 32, "int8", 3)


COUNTS = [37, 5, 20, 0, 100]
LENS = [60, 5, 12, 9, 100]                                      # (of the third one's rows 8 lie before token 0)


@pytest.mark.parametrize("max_rows", [1, 7, 16, 36])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_append_serves_the_first_rows_of_a_sequence(biq, fmt, max_rows):
    """Row i of n is token lens - n + i, whether or not the rows after it are served."""
    rng = np.random.default_rng(1)
    pages = su.Pages([112, 16, 32, 16, 112], 2, 64, 16, fmt, rng)
    pages.lens[:] = LENS
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((sum(COUNTS), 2, 64), generator=g) for _ in range(2))
    for s, (n, length) in enumerate(zip(COUNTS, LENS)):         # what was there before the call
        if length > n:
            pages.append(s, 0, rng.standard_normal((length - n, 2, 64)), rng.standard_normal((length - n, 2, 64)))
    cache = pages.on(biq)
    biq.biq_cache_append(cache, k.to("cuda:0"), v.to("cuda:0"), starts=au.starts_of(COUNTS), max_rows=max_rows)
    at = 0
    for s, n in enumerate(COUNTS):
        m = min(n, max_rows)
        pos, cut = LENS[s] - n, min(m, max(0, n - LENS[s]))     # rows before token 0 are dropped
        if m > cut:
            pages.append(s, pos + cut, k[at + cut:at + m].double().numpy(), v[at + cut:at + m].double().numpy())
        at += n
    got = cache.store.cpu().numpy()
    assert np.array_equal(got, pages.store), np.argwhere(got != pages.store)[:5]


@pytest.mark.parametrize("max_rows", [1, 7, 16, 36])
def test_read_serves_the_first_rows_of_a_sequence(biq, max_rows):
    pages = su.filled(LENS, 2, 64, 32, "int8", 2)
    out = [torch.full((sum(COUNTS), 2, 64), 9.0, device="cuda:0") for _ in range(2)]
    biq.biq_cache_read(pages.on(biq), *out, starts=au.starts_of(COUNTS), max_rows=max_rows)
    at = 0
    for s, n in enumerate(COUNTS):
        m = min(n, max_rows)
        for got, held in zip(out, pages.values(s)):
            want = np.concatenate([np.zeros((max(0, n - LENS[s]), 2, 64)), held[max(0, LENS[s] - n):]])[:m]
            assert np.array_equal(got[at:at + m].cpu().numpy(), want.astype(np.float32)), s
            assert (got[at + m:at + n] == 9).all()
        at += n


@pytest.mark.parametrize("max_rows", [1, 7, 16, 36])
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_serves_the_first_rows_of_a_sequence(biq, causal, window, max_rows):
    """(With and without the tokens shared by workgroups; the kernel for many rows below.)"""
    for lens, counts, qh, max_len in ((LENS, COUNTS, 4, 0), ([900, 700, 12, 9, 640], COUNTS, 4, 900), ([300] * 16, [40] * 16, 512, 0)):
        pages = held(tuple(lens), *((2, 64) if qh == 4 else (32, 16)))
        q = au.rows_like(counts, qh, pages.dim, "fp32", 4)
        how = dict(starts=au.starts_of(counts), max_len=max_len, causal=causal, window=window)
        out, lse = au.call(biq, pages.on(biq), q.to("cuda:0"), max_rows=max_rows, **how)
        out, lse = out.double().cpu(), lse.double().cpu()
        at = 0
        for s, n in enumerate(counts):
            m = min(n, max_rows)
            if s < 5 or s == 15:
                k, v = (torch.from_numpy(x) for x in pages.values(s))
                want, want_lse, size, vmax = au.softmax64(q[at:at + m].double(), k, v, pages.dim ** -0.5, lens[s] - n + torch.arange(m), causal, window)
                tol, tol_lse = au.bounds("fp32", want, size, vmax, lens[s])
                assert ((out[at:at + m] - want).abs() <= tol).all(), s
                empty = torch.isinf(want_lse)
                assert torch.equal(torch.isinf(lse[at:at + m]), empty)
                assert ((lse[at:at + m] - want_lse).abs() <= tol_lse)[~empty].all(), s
                assert torch.isnan(out[at + m:at + n]).all()    # the others are left as they were
            at += n
