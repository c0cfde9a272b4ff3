"""Probabilities of biq_logits from logits that are large beside their differences: what is lost depends on the differences."""
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


def call(biq, x, h):
    out = torch.full(x.shape, float("nan"), device="cuda:0")
    ws = torch.full((max(16, biq.biq_logits_workspace_bytes(*x.shape)),), 0xff, dtype=torch.uint8, device="cuda:0")
    biq.biq_logits(x.to("cuda:0"), out, probabilities=True, workspace=ws, **{k: torch.from_numpy(v).to("cuda:0") for k, v in h.items()})
    return su.back(out)


def check(x, h, got):
    """Relative, in units of 2^-24.  An exponent (to base 2) is z - max times 1 / temperature and log2 e: four roundings of these factors and
    their product, two of the difference and the result, of an exponent that is 1.45 times as large and counts ln 2 of that: 6 of z - max.
    Exponentials of the hardware 2 each, three of them; a sum in 32 bits of which 32 terms follow one another at most, then trees of 16 levels; a
    division and two products.  Logits that are changed (said before, biased) have three roundings of the largest number on the way, over the
    temperature, and move the row's sum by as much where they have weight.  Below 2^-126 nothing is promised."""
    z, greedy = su.logits(x.double().numpy(), **h)
    p = su.probabilities(z, greedy)
    t = h["temperature"].astype(np.float64)[:, None, None] if "temperature" in h else np.ones((x.shape[0], 1, 1))
    base = 6 * np.where(np.isfinite(z), z.max(axis=2, keepdims=True) - z, 0) + 2 * 3 + 32 + 16 + 4
    plain, _ = su.logits(x.double().numpy(), **{k: v for k, v in h.items() if k == "temperature"})
    changed = np.isfinite(z) & (z != plain)
    moved = np.where(changed, 3 * np.maximum(np.abs(x.double().numpy()) * 1.5, np.abs(z * t)) / t, 0)
    bound = p * 2.0 ** -24 * (base + moved + (p * moved).sum(axis=2, keepdims=True)) + 2.0 ** -126
    bad = ~(np.abs(got - p) <= bound)
    assert not bad.any(), (np.max(np.abs(got - p) / bound), bad.sum())


@pytest.mark.parametrize("seqs,rows,vocab", [(2, 1, 700), (2, 2, 8000), (2, 3, 16001), (3, 2, 32000), (2, 1, 150001), (128, 2, 20001)])
@pytest.mark.parametrize("middle", [0.0, 200.0, -1000.0, 30000.0, 1e6])
@pytest.mark.parametrize("heat", [1.0, 0.7])
def test_large_logits(biq, seqs, rows, vocab, middle, heat):
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn((seqs, rows, vocab), generator=g) * 3 + middle
    h = dict(temperature=np.full(seqs, heat, np.float32))
    check(x, h, call(biq, x, h))


@pytest.mark.parametrize("seqs,rows,vocab", [(2, 3, 700), (3, 3, 16001), (2, 3, 50001), (128, 2, 20001)])
@pytest.mark.parametrize("middle", [0.0, 1000.0])
def test_large_logits_of_tokens_said_before(biq, seqs, rows, vocab, middle):
    """Those said before are few beside the others, which keep their precision."""
    g = torch.Generator().manual_seed(vocab)
    rng = np.random.default_rng(vocab)
    x = torch.randn((seqs, rows, vocab), generator=g) * 3 + middle
    h = dict(history=rng.integers(0, vocab, size=(seqs, 30)).astype(np.int32), lens=np.full(seqs, 30, np.int32), prompt_lens=np.full(seqs, 10, np.int32),
             drafts=rng.integers(0, vocab, size=(seqs, rows - 1)).astype(np.int32), repetition=np.full(seqs, 1.01, np.float32),
             presence=np.full(seqs, 0.3, np.float32), frequency=np.full(seqs, 0.2, np.float32), temperature=np.full(seqs, 0.8, np.float32))
    check(x, h, call(biq, x, h))


@pytest.mark.parametrize("vocab", [900, 9001, 20001])
def test_cold_rows_of_large_logits(biq, vocab):
    """Exponents beyond 2^24, whose rounding alone would move probabilities: the differences count."""
    x = torch.full((4, 1, vocab), 1000.0)
    x[:, 0, [3, vocab - 1]] = 1001.0
    x[:, 0, 4] = np.nextafter(np.float32(1001), np.float32(0)).item()
    heat = np.array([1e-3, 1e-5, 1e-12, 1e-25], np.float32)
    p = call(biq, x, dict(temperature=heat))[:, 0]
    step = 1001.0 - x[0, 0, 4].item()
    for s in range(4):
        least = np.exp(-step / float(heat[s]))
        want = np.zeros(vocab)
        want[[3, vocab - 1]], want[4] = 1, least
        want /= want.sum()
        assert (np.abs(p[s] - want) <= 2.0 ** -24 * (64 + 6 * min(step / float(heat[s]), 100)) * want + 2.0 ** -126).all(), s
