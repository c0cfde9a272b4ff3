"""The operators at the end of a decoder step one after the other, as they are used; captured, on other streams, and twice at once."""
import os
import sys

import numpy as np
import pytest
import torch

import step_util as su

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


class Chain:
    """norm -> 4-bit head on its codes -> logits -> verification, all buffers held."""

    def __init__(self, biq, seqs, drafts, hidden, vocab, group=128, fmt="int8", stream=None, seed=0):
        g = torch.Generator().manual_seed(seed)
        rows = seqs * (drafts + 1)
        self.x, self.res = (torch.randn((rows, hidden), generator=g).bfloat16().to(DEV) for _ in range(2))
        self.weight = (1 + 0.2 * torch.randn(hidden, generator=g)).to(DEV)
        self.W = torch.randn((vocab, hidden), generator=g) * hidden ** -0.5 * 3
        self.packed = torch.empty(biq.biq_packed4_bytes(vocab, hidden, group), dtype=torch.uint8, device=DEV)
        biq.biq_quantize4(self.W.to(DEV), self.packed, vocab, hidden, group)
        self.sum = torch.empty_like(self.x)
        self.codes = torch.empty((rows, hidden), dtype=torch.int8 if fmt == "int8" else torch.float8_e4m3fn, device=DEV)
        self.scales = torch.empty((rows, su.groups(hidden, group)), device=DEV)
        self.z = torch.empty((rows, vocab), device=DEV)
        self.p = torch.empty((seqs, drafts + 1, vocab), device=DEV)
        self.drafts = torch.randint(0, vocab, (seqs, drafts), generator=g, dtype=torch.int32).to(DEV)
        self.history = torch.randint(0, vocab, (seqs, 50), generator=g, dtype=torch.int32).to(DEV)
        self.lens = torch.randint(1, 51, (seqs,), generator=g, dtype=torch.int32).to(DEV)
        self.penalty = torch.full((seqs,), 1.2, device=DEV)
        self.uniform = torch.rand((seqs, drafts + 1), generator=g).to(DEV)
        self.tokens = torch.empty((seqs, drafts + 1), dtype=torch.int32, device=DEV)
        self.accepted = torch.empty(seqs, dtype=torch.int32, device=DEV)
        space = lambda n: torch.empty(max(16, n), dtype=torch.uint8, device=DEV)
        how = dict(x_scales=self.scales, x_group=group)
        self.group, self.seqs, self.drafts_n = group, seqs, drafts
        self.calls = [
            biq.PreparedNorm(self.x, weight=self.weight, residual=self.res, sum=self.sum, codes=self.codes, scales=self.scales, group=group, stream=stream),
            biq.PreparedGemm4(self.packed, self.codes, self.z, group, workspace=space(biq.biq_gemm4_workspace_bytes(self.packed, self.codes, self.z, group, **how)),
                              stream=stream, **how),
            biq.PreparedLogits(self.z.view(seqs, drafts + 1, vocab), self.p, history=self.history, lens=self.lens, drafts=self.drafts, repetition=self.penalty,
                               probabilities=True, workspace=space(biq.biq_logits_workspace_bytes(seqs, drafts + 1, vocab)), stream=stream),
            biq.PreparedVerify(self.p, None, self.drafts, self.uniform, self.tokens, self.accepted,
                               workspace=space(biq.biq_verify_workspace_bytes(seqs, vocab)), stream=stream)]

    def __call__(self):
        for call in self.calls:
            call()

    def results(self):
        return [t.clone() for t in (self.sum, self.codes.float(), self.scales, self.z, self.p, self.tokens, self.accepted)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("seqs,drafts,hidden,vocab,fmt", [(1, 0, 256, 1000, "int8"), (4, 3, 1000, 5003, "int8"), (9, 4, 640, 20001, "fp8")])
def test_against_64_bits(biq, seqs, drafts, hidden, vocab, fmt):
    """On the codes that were written: the product as its own test bounds it (2^-21 of the magnitudes' sums in the mean, taken four times for single
    elements here), and probabilities moved by twice the product's error."""
    c = Chain(biq, seqs, drafts, hidden, vocab, fmt=fmt)
    c()
    x, res = (t.float().cpu().numpy() for t in (c.x, c.res))
    codes, units = su.norm_codes(x, res, c.weight.cpu().numpy(), 0.0, c.group, fmt)
    assert np.array_equal(su.back(c.codes.float()), codes)
    held = codes * su.spread(su.back(c.scales), hidden, c.group)
    w4, ws = su.quantized4(c.W.numpy(), c.group)
    w = w4 * su.spread(ws.astype(np.float64), hidden, c.group)
    z, size = held @ w.T, np.abs(held) @ np.abs(w).T
    assert (np.abs(su.back(c.z) - z) <= 2.0 ** -19 * size).all()
    adjusted, greedy = su.logits(z.reshape(seqs, drafts + 1, vocab), history=c.history.cpu().numpy(), lens=c.lens.cpu().numpy(), drafts=c.drafts.cpu().numpy(),
                                 repetition=c.penalty.cpu().numpy())
    p = su.probabilities(adjusted, greedy)
    assert (np.abs(su.back(c.p) - p) <= p * (2.0 ** -17 * size.max() * 1.2 + 2.0 ** -17) + 2.0 ** -25).all()


def test_captured_and_replayed(biq):
    """A graph of the chain, replayed with eager work and synchronizations between; inputs change in place."""
    c = Chain(biq, 5, 3, 512, 20001, seed=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held = Chain(biq, 5, 3, 512, 20001, seed=1)
        held()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held()
    for step in range(4):
        for chain in (c, held):
            chain.x.mul_(1.25)
            chain.history.add_(1)
            chain.uniform.mul_(0.9)
        c()
        for t in (held.z, held.p, held.sum):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert same(c.results(), held.results()), step
        torch.randn(1000, device=DEV).sum().item()


def test_two_streams_at_once(biq):
    """Two chains with buffers of their own on two streams give what each gives alone."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    chains = [Chain(biq, 6, 2, 768, 9001, stream=s, seed=7 + i) for i, s in enumerate(streams)]
    torch.cuda.synchronize()
    alone = []
    for c in chains:
        c()
        torch.cuda.synchronize()
        alone.append(c.results())
    for _ in range(10):
        for c in chains:
            for t in (c.z, c.p):
                t.zero_()
        torch.cuda.synchronize()
        for c in chains:
            c()
        torch.cuda.synchronize()
        assert all(same(c.results(), a) for c, a in zip(chains, alone))


def test_an_example_whose_prompts_begin_alike(biq):
    """Shared pages and separate ones give the same tokens, but for what rounding of the caches' codes may turn: where a token of the beginning lies in a
    block with later ones it is rounded anew, and no whole page of the beginning has such a block."""
    import speculative_decode as ex

    model = ex.Decoder(hidden=256, heads=4, kv_heads=2, dim=64, ffn=512, layers=2, vocab=333, planes=3, positions=512)
    beginning, prompts = [(7 * i) % 333 for i in range(150)], [[1, 2, 3], [9], list(range(20))]
    together = ex.answer_alike(model, beginning, prompts, 12)
    assert all(len(a) == 12 and all(0 <= t < 333 for t in a) for a in together)
    whole = ex.answer_alike(model, [], [beginning + p for p in prompts], 12)
    agree = [np.mean([x == y for x, y in zip(a, b)]) for a, b in zip(together, whole)]
    assert all(a[0] == b[0] for a, b in zip(together, whole)) and np.mean(agree) > 0.5, agree
