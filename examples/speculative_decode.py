"""A small decoder on binary-coded weights that drafts its own tokens: its first bit-planes are a cheaper, rougher model of the
same function, and packed planes lie one after the other, so the draft model is the target's matrices with fewer planes.

Every step runs on the library's kernels: biq_norm with the residual's addition, biq_gemm for the projections, biq_rotary and
biq_cache_append for queries and keys, biq_attention over the paged 8-bit cache, biq_gemm4 for the output head in 4 bits, on the last norm's
codes, biq_logits for probabilities, biq_verify_drafts for the drafts and for drawing tokens (torch does the embedding's lookup and
activations).  Prompts that begin alike can have the beginning's pages in common (answer_alike): biq_attention_shared reads
them once for all sequences.  Weights are random: what is shown is how the calls fit together.

    python examples/speculative_decode.py [--tokens 32] [--drafts 4] [--planes 3] [--draft-planes 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2005_09904_amd as biq

MU, PAGE = 8, 64


class Linear:
    """A binary-coded matrix [m][n]: packed signs and scales of all planes."""

    def __init__(self, m, n, planes, g, device):
        w = torch.randn((m, n), device=device, generator=g) * n ** -0.5
        self.m, self.n = m, n
        self.K = torch.empty(biq.biq_packed_bytes(m, n, planes), dtype=torch.uint8, device=device)
        self.alpha = torch.empty((planes, m), device=device)
        biq.biq_quantize(w, self.K, self.alpha, m, n, planes)

    def __call__(self, x, planes):
        """x [rows, n] -> [rows, m] with the first planes."""
        y = torch.empty((x.shape[0], self.m), device=x.device)
        ws = torch.empty(max(16, biq.biq_workspace_bytes(self.m, self.n, planes, x.shape[0], MU)), dtype=torch.uint8, device=x.device)
        biq.biq_gemm(self.K, self.alpha, x.contiguous(), y, self.m, self.n, planes, x.shape[0], MU, workspace=ws)
        return y


class Linear4:
    """A matrix [m][n] in 4 bits for inputs in 8 bits, both with a scale for 128 elements: the output head, which binary codes serve worst."""

    GROUP = 128

    def __init__(self, m, n, g, device):
        self.m, self.n = m, n
        self.packed = torch.empty(biq.biq_packed4_bytes(m, n, self.GROUP), dtype=torch.uint8, device=device)
        biq.biq_quantize4(torch.randn((m, n), device=device, generator=g) * n ** -0.5, self.packed, m, n, self.GROUP)

    def __call__(self, codes, scales):
        y = torch.empty((codes.shape[0], self.m), device=codes.device)
        how = dict(x_scales=scales, x_group=self.GROUP)
        ws = torch.empty(max(16, biq.biq_gemm4_workspace_bytes(self.packed, codes, y, self.GROUP, **how)), dtype=torch.uint8, device=codes.device)
        biq.biq_gemm4(self.packed, codes, y, self.GROUP, workspace=ws, **how)
        return y


class Decoder:
    def __init__(self, hidden=512, heads=8, kv_heads=2, dim=64, ffn=1024, layers=2, vocab=1000, planes=3, positions=2048, seed=0,
                 device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.hidden, self.heads, self.kv_heads, self.dim, self.ffn, self.vocab, self.planes = hidden, heads, kv_heads, dim, ffn, vocab, planes
        self.embedding = torch.randn((vocab, hidden), device=device, generator=g)
        self.layers = [dict(qkv=Linear((heads + 2 * kv_heads) * dim, hidden, planes, g, device), out=Linear(hidden, heads * dim, planes, g, device),
                            up=Linear(2 * ffn, hidden, planes, g, device), down=Linear(hidden, ffn, planes, g, device)) for _ in range(layers)]
        self.head = Linear4(vocab, hidden, g, device)
        self.angles = torch.empty((positions, dim // 2, 2), device=device)
        biq.biq_rotary_table(biq.biq_rotary_frequencies(dim, 10000.0, "linear", 2.0).to(device), self.angles)
        self.device, self.positions = device, positions

    def caches(self, seqs, format="int8", shared=0):
        """One paged cache per layer for that many sequences, all with the same lengths; the first `shared` tokens in the first one's pages."""
        per_seq = -(-self.positions // PAGE)
        lens = torch.zeros(seqs, dtype=torch.int32, device=self.device)
        table = torch.arange(seqs * per_seq, dtype=torch.int32, device=self.device).view(seqs, per_seq)
        table[:, :shared // PAGE] = table[0, :shared // PAGE].clone()
        page = biq.biq_cache_page_bytes(PAGE, self.kv_heads, self.dim)
        return [biq.KvCache(torch.zeros((seqs * per_seq, page), dtype=torch.uint8, device=self.device), table, lens, PAGE, self.kv_heads,
                            self.dim, format) for _ in self.layers]

    def forward(self, tokens, caches, planes, starts=None, max_rows=None, max_len=0, shared=0):
        """Probabilities [rows, vocab] of what follows each of the rows' tokens [rows].  The caches' lens have them counted already.  shared: tokens
        that all sequences begin with, in the first one's pages."""
        lens = caches[0].lens
        rows = tokens.shape[0]
        if starts is None:
            n = rows // lens.shape[0]
            pos = (lens[:, None] - n + torch.arange(n, dtype=torch.int32, device=self.device)).reshape(-1).contiguous()
        else:
            seq = torch.bucketize(torch.arange(rows, device=self.device), starts[1:].long(), right=True)
            pos = (torch.arange(rows, device=self.device) - starts[seq + 1] + lens[seq]).int()
        x = self.embedding[tokens.long()]
        y = torch.empty_like(x)
        biq.biq_norm(x, y)
        h, kv = self.heads, self.kv_heads
        for layer, cache in zip(self.layers, caches):
            qkv = layer["qkv"](y, planes).view(rows, h + 2 * kv, self.dim)
            q, k, v = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
            biq.biq_rotary(q, q, pos, self.angles)
            biq.biq_cache_append(cache, k, v, starts=starts, max_rows=max_rows, angles=self.angles)
            out = torch.empty((rows, h, self.dim), device=self.device)
            how = dict(starts=starts, max_rows=max_rows, max_len=max_len)
            if shared:
                ws = torch.empty(biq.biq_attention_shared_workspace_bytes(cache, q, shared, **how), dtype=torch.uint8, device=self.device)
                biq.biq_attention_shared(cache, q, out, shared, workspace=ws, **how)
            else:
                ws = torch.empty(max(16, biq.biq_attention_workspace_bytes(cache, q, **how)), dtype=torch.uint8, device=self.device)
                biq.biq_attention(cache, q, out, workspace=ws, **how)
            biq.biq_norm(layer["out"](out.view(rows, -1), planes), y, residual=x, sum=x)
            up = layer["up"](y, planes)
            down = layer["down"](torch.nn.functional.silu(up[:, :self.ffn]) * up[:, self.ffn:], planes)
            if layer is not self.layers[-1]:
                biq.biq_norm(down, y, residual=x, sum=x)
        # the last norm's result is wanted in 8 bits
        codes = torch.empty((rows, self.hidden), dtype=torch.int8, device=self.device)
        scales = torch.empty((rows, -(-self.hidden // Linear4.GROUP)), device=self.device)
        biq.biq_norm(down, residual=x, codes=codes, scales=scales, group=Linear4.GROUP)
        z = self.head(codes, scales)[:, None]
        ws = torch.empty(max(16, biq.biq_logits_workspace_bytes(rows, 1, self.vocab)), dtype=torch.uint8, device=self.device)
        biq.biq_logits(z, z, probabilities=True, workspace=ws)
        return z[:, 0]


def draw(p, u):
    """A token of every row of p [seqs, vocab] by the numbers u [seqs]."""
    seqs, vocab = p.shape
    tokens, none = torch.empty((seqs, 1), dtype=torch.int32, device=p.device), torch.empty(seqs, dtype=torch.int32, device=p.device)
    ws = torch.empty(biq.biq_verify_workspace_bytes(seqs, vocab), dtype=torch.uint8, device=p.device)
    biq.biq_verify_drafts(p[:, None], None, torch.empty((seqs, 0), dtype=torch.int32, device=p.device), u[:, None].contiguous(), tokens, none,
                          workspace=ws)
    return tokens[:, 0]


def generate(model, prompts, tokens, drafts=4, draft_planes=2, seed=0, format="int8"):
    """Continues prompts (lists of token numbers); returns the tokens of every sequence and the share of drafts accepted."""
    dev, seqs, vocab = model.device, len(prompts), model.vocab
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    counts = [len(p) for p in prompts]
    starts = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device=dev)
    flat = torch.tensor([t for p in prompts for t in p], dtype=torch.int32, device=dev)
    target, draft = model.caches(seqs, format), model.caches(seqs, format)
    for caches, planes in ((draft, draft_planes), (target, model.planes)):
        caches[0].lens.copy_(torch.diff(starts))               # (one tensor for all layers)
        p = model.forward(flat, caches, planes, starts, max(counts), max(counts))
    last = draw(p[starts[1:].long() - 1], torch.rand(seqs, device=dev, generator=g))
    answers = [[t] for t in last.tolist()]
    ws = torch.empty(biq.biq_verify_workspace_bytes(seqs, vocab), dtype=torch.uint8, device=dev)
    accepted_all = offered = 0
    longest = max(counts)
    while min(len(a) for a in answers) < tokens:
        longest += drafts + 1
        # the draft model writes one token after the other (the last of them only for its cache)
        q = torch.empty((seqs, drafts, vocab), device=dev)
        fed = torch.empty((seqs, drafts + 1), dtype=torch.int32, device=dev)
        fed[:, 0] = last
        for i in range(drafts + 1):
            draft[0].lens.add_(1)
            probs = model.forward(fed[:, i].contiguous(), draft, draft_planes, max_len=longest)
            if i < drafts:
                q[:, i] = probs
                fed[:, i + 1] = draw(probs, torch.rand(seqs, device=dev, generator=g))
        # the target sees them all at once
        target[0].lens.add_(drafts + 1)
        p = model.forward(fed.reshape(-1), target, model.planes, max_len=longest).view(seqs, drafts + 1, vocab)
        out, accepted = torch.empty_like(fed), torch.empty(seqs, dtype=torch.int32, device=dev)
        biq.biq_verify_drafts(p, q, fed[:, 1:].contiguous(), torch.rand((seqs, drafts + 1), device=dev, generator=g), out, accepted, workspace=ws)
        # what was not accepted leaves both caches
        for caches in (target, draft):
            caches[0].lens.add_(accepted - drafts)
        last = out.gather(1, accepted.long()[:, None])[:, 0]
        for s, (n, row) in enumerate(zip(accepted.tolist(), out.tolist())):
            answers[s] += row[:n + 1]
            accepted_all += n
            offered += drafts
    return answers, accepted_all / max(offered, 1), target, draft


def answer_alike(model, beginning, prompts, tokens, seed=0):
    """Continues prompts that all begin with the tokens `beginning`, whose whole pages are written once and read once for all of them."""
    dev, seqs = model.device, len(prompts)
    shared = len(beginning) // PAGE * PAGE
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    caches = model.caches(seqs, shared=shared)
    lens = caches[0].lens
    if shared:                                                  # rows of the first sequence alone
        lens[0] = shared
        rows = [0] + [shared] * seqs
        model.forward(torch.tensor(beginning[:shared], dtype=torch.int32, device=dev), caches, model.planes,
                      torch.tensor(rows, dtype=torch.int32, device=dev), shared, shared)
    rest = [beginning[shared:] + p for p in prompts]
    starts = torch.tensor([0, *torch.tensor([len(p) for p in rest]).cumsum(0).tolist()], dtype=torch.int32, device=dev)
    longest = shared + max(map(len, rest))
    lens.copy_(shared + torch.diff(starts))
    p = model.forward(torch.tensor([t for r in rest for t in r], dtype=torch.int32, device=dev), caches, model.planes, starts, max(map(len, rest)), longest,
                      shared)
    last = draw(p[starts[1:].long() - 1], torch.rand(seqs, device=dev, generator=g))
    answers = [last]
    for _ in range(tokens - 1):
        lens.add_(1)
        longest += 1
        last = draw(model.forward(last.contiguous(), caches, model.planes, max_len=longest, shared=shared), torch.rand(seqs, device=dev, generator=g))
        answers.append(last)
    return torch.stack(answers, dim=1).tolist()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--planes", type=int, default=3)
    ap.add_argument("--draft-planes", type=int, default=2)
    a = ap.parse_args()
    model = Decoder(planes=a.planes)
    answers, rate, _, _ = generate(model, [[1, 2, 3, 4, 5], [7] * 90, [11]], a.tokens, a.drafts, a.draft_planes)
    for s, t in enumerate(answers):
        print("sequence %d: %s" % (s, " ".join(map(str, t))))
    print("%.0f %% of the drafts accepted" % (100 * rate))
    for s, t in enumerate(answer_alike(model, [5] * 100, [[1, 2], [3], [4] * 9], a.tokens)):
        print("answer %d to prompts that begin alike: %s" % (s, " ".join(map(str, t))))


if __name__ == "__main__":
    main()
