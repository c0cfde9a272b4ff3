"""bf16 outputs of biq_attention_shared are off by their own rounding alone: weights, like sums, are held in more bits."""
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


def constant_values(shared, lens, heads, dim, page):
    """All tokens have, in head h, one value: beside the middle of two bf16 numbers, by 2^-13 to either side, as a code of 64 + 4 h.  Their keys are one
    too, but for the first token's of every block, which is three times that."""
    pages = su.Pages([max(lens[0], shared), *lens[1:]], heads, dim, page, "int8", np.random.default_rng(dim))
    pages.lens[0] = lens[0]
    keys = np.full((su.BLOCK, dim), 16.0 * (1 - 2 * (np.arange(dim) % 2)))
    keys[0] *= 3
    for s, n in enumerate(lens):
        for b in range(-(-(n if s else max(n, shared)) // su.BLOCK)):
            for h in range(heads):
                code = 64 + 4 * h
                value = 1 + 2.0 ** -8 + (2.0 ** -13 if h % 2 else -2.0 ** -13)
                pages.put(s, b, h, 0, keys, np.float32(2.0 ** -9))
                pages.put(s, b, h, 1, np.full((su.BLOCK, dim), float(code)), np.float32(value / code))
    pages.table[1:, :shared // page] = pages.table[0, :shared // page]
    return pages


@pytest.mark.parametrize("dim", [48, 64, 128, 192, 256])
@pytest.mark.parametrize("new,max_rows", [(1, 1), (5, 5), (70, 70), (9, 80)])
def test_bf16_outputs_round_once(biq, dim, new, max_rows):
    """A mean of equal values is the value.  What their weights and sums may cost is that of 32-bit outputs: 2^-22 a weight, units of 32 bits for
    scores, sums and steps."""
    heads, shared, lens = 16, 192, (193 + new, 300 + new, 192 + new, 250 + new)
    pages = constant_values(shared, lens, heads, dim, 32)
    q = au.rows_like([new] * 4, heads, dim, "bf16", new + dim, 1.0).to("cuda:0")
    cache = pages.on(biq)
    how = dict(starts=au.starts_of([new] * 4), max_rows=max_rows, max_len=max(lens))
    out = torch.full_like(q, float("nan"))
    ws = torch.full((biq.biq_attention_shared_workspace_bytes(cache, q, shared, **how),), 0xff, dtype=torch.uint8, device="cuda:0")
    biq.biq_attention_shared(cache, q, out, shared, workspace=ws, **how)
    value = torch.from_numpy(pages.values(1)[1][0])                                 # [heads][dim]
    size = dim ** -0.5 * 3 * 2.0 ** -5 * q.double().abs().sum(dim=2).max().item()
    slack = 2 * (2.0 ** -24 * (8 * size + 16 + (2 * max(lens) + 128) / 64) + 2.0 ** -22 + max(lens) * 2.0 ** -38) * 1.01
    assert slack < 2.0 ** -15                                                       # (far less than the values' distance from the middle)
    off = (out.double().cpu() - value).abs()
    assert (off <= 2.0 ** -8 + slack).all(), (off.max().item(), (off > 2.0 ** -8 + slack).any(dim=2).sum(dim=0).tolist())
