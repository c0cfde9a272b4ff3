"""A small decoder on binary-coded weights that drafts its own tokens: its first bit-planes are a cheaper, rougher model of the
same function, and packed planes lie one after the other, so the draft model is the target's matrices with fewer planes.

Every step runs on the library's kernels: biq_gemm for the projections, biq_rotary and biq_cache_append for queries and
keys, biq_attention over the paged 8-bit cache, biq_verify_drafts for the drafts and for drawing tokens (torch does norms,
activations and the softmax over the vocabulary).  Weights are random: what is shown is how the calls fit together.

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


class Decoder:
    def __init__(self, hidden=512, heads=8, kv_heads=2, dim=64, ffn=1024, layers=2, vocab=1000, planes=3, positions=2048, seed=0,
                 device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.hidden, self.heads, self.kv_heads, self.dim, self.ffn, self.vocab, self.planes = hidden, heads, kv_heads, dim, ffn, vocab, planes
        self.embedding = torch.randn((vocab, hidden), device=device, generator=g)
        self.layers = [dict(qkv=Linear((heads + 2 * kv_heads) * dim, hidden, planes, g, device), out=Linear(hidden, heads * dim, planes, g, device),
                            up=Linear(2 * ffn, hidden, planes, g, device), down=Linear(hidden, ffn, planes, g, device)) for _ in range(layers)]
        self.head = Linear(vocab, hidden, planes, g, device)
        self.angles = torch.empty((positions, dim // 2, 2), device=device)
        biq.biq_rotary_table(biq.biq_rotary_frequencies(dim, 10000.0, "linear", 2.0).to(device), self.angles)
        self.device, self.positions = device, positions

    def caches(self, seqs, format="int8"):
        """One paged cache per layer for that many sequences, all with the same lengths."""
        per_seq = -(-self.positions // PAGE)
        lens = torch.zeros(seqs, dtype=torch.int32, device=self.device)
        table = torch.arange(seqs * per_seq, dtype=torch.int32, device=self.device).view(seqs, per_seq)
        page = biq.biq_cache_page_bytes(PAGE, self.kv_heads, self.dim)
        return [biq.KvCache(torch.zeros((seqs * per_seq, page), dtype=torch.uint8, device=self.device), table, lens, PAGE, self.kv_heads,
                            self.dim, format) for _ in self.layers]

    def forward(self, tokens, caches, planes, starts=None, max_rows=None, max_len=0):
        """Probabilities [rows, vocab] of what follows each of the rows' tokens [rows].  The caches' lens have them counted already."""
        lens = caches[0].lens
        rows = tokens.shape[0]
        if starts is None:
            n = rows // lens.shape[0]
            pos = (lens[:, None] - n + torch.arange(n, dtype=torch.int32, device=self.device)).reshape(-1).contiguous()
        else:
            seq = torch.bucketize(torch.arange(rows, device=self.device), starts[1:].long(), right=True)
            pos = (torch.arange(rows, device=self.device) - starts[seq + 1] + lens[seq]).int()
        x = self.embedding[tokens.long()]
        norm = lambda t: t * torch.rsqrt(t.square().mean(dim=1, keepdim=True) + 1e-6)
        h, kv = self.heads, self.kv_heads
        for layer, cache in zip(self.layers, caches):
            qkv = layer["qkv"](norm(x), planes).view(rows, h + 2 * kv, self.dim)
            q, k, v = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
            biq.biq_rotary(q, q, pos, self.angles)
            biq.biq_cache_append(cache, k, v, starts=starts, max_rows=max_rows, angles=self.angles)
            out = torch.empty((rows, h, self.dim), device=self.device)
            how = dict(starts=starts, max_rows=max_rows, max_len=max_len)
            ws = torch.empty(max(16, biq.biq_attention_workspace_bytes(cache, q, **how)), dtype=torch.uint8, device=self.device)
            biq.biq_attention(cache, q, out, workspace=ws, **how)
            x = x + layer["out"](out.view(rows, -1), planes)
            up = layer["up"](norm(x), planes)
            x = x + layer["down"](torch.nn.functional.silu(up[:, :self.ffn]) * up[:, self.ffn:], planes)
        return torch.softmax(self.head(norm(x), planes), dim=1)


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


if __name__ == "__main__":
    main()
