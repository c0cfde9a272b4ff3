"""biq_attention against softmax in 64 bits, whole matrices at a time, with bounds that grow with the values' magnitude."""
import numpy as np
import torch

import serving_util as su


def call(biq, cache, q, **how):
    """Output and lse of a call whose buffers are poisoned."""
    ws = torch.full((max(16, biq.biq_attention_workspace_bytes(cache, q, **how)),), 0xff, dtype=torch.uint8, device=q.device)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device=q.device)
    lse = torch.full(q.shape[:2], float("nan"), device=q.device)
    biq.biq_attention(cache, q, out, lse=lse, workspace=ws, **how)
    torch.cuda.synchronize()
    return out, lse


def softmax64(q, k, v, scale, pos, causal, window):
    """q [rows][qh][dim], k, v [len][heads][dim] (CPU, 64 bits), pos [rows] -> out, lse, the largest sum of |scale q k|, the largest |v|."""
    rows, qh, dim = q.shape
    length, heads = k.shape[:2]
    out, lse = torch.zeros((rows, qh, dim), dtype=torch.float64), torch.full((rows, qh), float("-inf"), dtype=torch.float64)
    size = 0.0
    t = torch.arange(length)
    hidden = torch.zeros((rows, length), dtype=torch.bool)
    if causal:
        hidden |= t[None, :] > pos[:, None]
    if window:
        hidden |= t[None, :] <= pos[:, None] - window
    some = ~hidden.all(dim=1)
    for h in range(qh):
        kh, vh = k[:, h // (qh // heads)], v[:, h // (qh // heads)]
        z = (scale * (q[:, h] @ kh.T)).masked_fill_(hidden, float("-inf"))
        if not some.any():
            continue
        size = max(size, (abs(scale) * (q[:, h].abs() @ kh.abs().T)).masked_fill_(hidden, 0.0).max().item())
        m = z[some].amax(dim=1, keepdim=True)
        e = torch.exp(z[some] - m)
        lse[some, h] = (m + torch.log(e.sum(dim=1, keepdim=True)))[:, 0]
        out[some, h] = e @ vh / e.sum(dim=1, keepdim=True)
    return out, lse, size, v.abs().max().item() if length else 0.0


def bounds(typ, out, size, vmax, length):
    """What rounding may cost.  Scores: rows of 32 bits are two 16-bit floats (2^-23 of them is lost), sums over a head in 32 bits (8
    units of the largest sum of magnitudes, eight times what a sum of 128 random signs has), one product and the exponential: a relative
    error of the weights, and an absolute one of the log-sum.  Sums over the tokens in 32 bits: a unit for every step of 64.  Weights: two
    16-bit floats (2^-22), one for bf16 (2^-11), and those below 2^-38 of the largest are lost.  A weight that is off by a relative e moves a
    mean of values by at most 2 e times the largest.  Then the output's own rounding, and its least number for fp16."""
    e = 2.0 ** -24 * (8 * size + 16 + length / 64)
    weight = {"fp32": 2.0 ** -22, "fp16": 2.0 ** -22, "bf16": 2.0 ** -11}[typ] + length * 2.0 ** -38
    own = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}[typ]
    return 2 * (e + weight) * vmax + own * out.abs() + (2.0 ** -25 if typ == "fp16" else 0.0), e + 2.0 ** -22 * (1 + size)


def rows_like(counts, qh, dim, typ, seed, big=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((sum(counts), qh, dim), generator=g) * big).to(su.TYPES[typ])


def starts_of(counts):
    return torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda:0")


def check(biq, pages, counts, q, typ, causal=True, window=0, scale=None, sample=None, **how):
    """A ragged call against 64 bits; sample: rows of every sequence that are looked at (all of them otherwise)."""
    how = {"max_rows": max(counts), **how}
    scale = pages.dim ** -0.5 if scale is None else scale
    out, lse = call(biq, pages.on(biq), q.to("cuda:0"), causal=causal, window=window, scale=scale, starts=starts_of(counts), **how)
    out, lse = out.double().cpu(), lse.double().cpu()
    at = 0
    for s, n in enumerate(counts):
        length = int(pages.lens[s])
        pick = torch.arange(n) if sample is None else torch.tensor(sorted({r % n for r in sample} if n else set()), dtype=torch.int64)
        k, v = (torch.from_numpy(x) for x in pages.values(s))
        want, want_lse, size, vmax = softmax64(q[at + pick].double(), k, v, scale, length - n + pick, causal, window)
        tol, tol_lse = bounds(typ, want, size, vmax, length)
        got, got_lse = out[at + pick], lse[at + pick]
        bad = ~((got - want).abs() <= tol)
        assert not bad.any(), (s, n, length, ((got - want).abs() / tol).max().item(), bad.sum().item(), bad.nonzero()[0].tolist())
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(got_lse), empty) and (got[empty] == 0).all()
        bad = ~((got_lse - want_lse).abs() <= tol_lse) & ~empty
        assert not bad.any(), (s, n, length, got_lse[bad][:3].tolist(), want_lse[bad][:3].tolist(), tol_lse)
        at += n
    return out, lse
