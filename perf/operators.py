"""The operators of a decoder step that stand beside the multiply, as cases that can be timed and checked: rotary
positions, the paged 8-bit cache's writer, attention over that cache, verification of drafted tokens.

A case is one call of a public entry point (the writer's: the call and a read of what it changed).  `run` makes it, or,
where `own` is false, computes the same in elementary torch operations in 32 bits.  Sizes are generic.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 16                                    # tokens that share a scale


def listed():
    return [
        # -- attention over the cache -------------------------------------------------------------------
        # a first answer's token of one short sequence: latency and little else
        dict(name="attn_token_short", kind="attn", seqs=1, new=1, len=77, ragged=False, qh=8, heads=8, dim=64, page=16,
             fmt="int8", type="fp32", causal=True, window=0),
        # an ordinary decoding step of a serving batch, lengths as they come
        dict(name="attn_token_b32", kind="attn", seqs=32, new=1, len=4096, ragged=True, qh=32, heads=8, dim=128, page=64,
             fmt="int8", type="fp32", causal=True, window=0),
        # a token of one very long conversation: the cache's bytes bound it, and the axis has to be split
        dict(name="attn_token_long", kind="attn", seqs=1, new=1, len=131071, ragged=False, qh=32, heads=8, dim=128,
             page=128, fmt="fp8", type="bf16", causal=True, window=0),
        # four drafted tokens and the one before them, to be verified in one pass
        dict(name="attn_drafts_b16", kind="attn", seqs=16, new=5, len=8192, ragged=True, qh=32, heads=8, dim=128, page=64,
             fmt="int8", type="bf16", causal=True, window=0),
        # the second half of long prompts over what the first half left in the cache
        dict(name="attn_prompt_b2", kind="attn", seqs=2, new=4096, len=8192, ragged=False, qh=32, heads=8, dim=128, page=64,
             fmt="int8", type="bf16", causal=True, window=0),
        # ragged prompts under a sliding window, an odd head size, pages that end inside a tile
        dict(name="attn_prompt_window", kind="attn", seqs=6, new=1500, len=2500, ragged=True, qh=20, heads=4, dim=80,
             page=48, fmt="fp8", type="fp32", causal=True, window=1024),
        # -- the cache's writer (keys rotated on the way) --------------------------------------------------
        # a decoding step of a large serving batch
        dict(name="append_token_b64", kind="append", seqs=64, new=1, len=2000, ragged=True, heads=8, dim=128, page=64,
             fmt="int8", type="fp32", rot=128, interleaved=False),
        # prompts as they come in, half the head rotated
        dict(name="append_prompt_b4", kind="append", seqs=4, new=4096, len=4500, ragged=True, heads=8, dim=128, page=64,
             fmt="fp8", type="bf16", rot=64, interleaved=True),
        # -- rotary positions -----------------------------------------------------------------------------
        # queries and keys of a decoding step, adjacent in the projection's output
        dict(name="rotary_token_b8", kind="rotary", rows=8, heads=40, dim=128, rot=128, interleaved=False, type="fp32",
             inverse=False, max_pos=32768),
        # the gradient of a training batch's queries and keys
        dict(name="rotary_prompt_grad", kind="rotary", rows=16384, heads=40, dim=128, rot=128, interleaved=True, type="bf16",
             inverse=True, max_pos=32768),
        # -- verification of drafted tokens ----------------------------------------------------------------
        # one sequence, four drafts, a small vocabulary
        dict(name="verify_b1", kind="verify", seqs=1, drafts=4, vocab=32000, type="fp32", draft_probs=True),
        # a serving batch with a large vocabulary of an odd size
        dict(name="verify_b64", kind="verify", seqs=64, drafts=7, vocab=120011, type="fp32", draft_probs=True),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm of [lo, hi], odd values among them."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.3 and v >= 64:
        v = v // 64 * 64
    v = max(lo, min(hi, v))
    return v + 1 if v == 3072 else v


def draw(rng):
    kind = rng.choice(["attn"] * 6 + ["append"] * 2 + ["rotary"] * 2 + ["verify"] * 2)
    typ = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if kind == "rotary":
        dim = 16 * rng.randint(2, 16)
        return dict(kind=kind, rows=_log_int(rng, 1, 16384), heads=rng.randint(1, 40), dim=dim,
                    rot=rng.choice([dim, dim // 2, 2 * rng.randint(1, dim // 2)]), interleaved=rng.random() < 0.5,
                    type=typ, inverse=rng.random() < 0.5, max_pos=32768) | ({"dim": 128, "rot": 128} if rng.random() < 0.3 else {})
    if kind == "verify":
        seqs = _log_int(rng, 1, 64)
        return dict(kind=kind, seqs=seqs, drafts=rng.randint(1, 7), vocab=_log_int(rng, 1000, 120000),
                    type=typ, draft_probs=rng.random() < 0.8)
    heads = rng.choice([1, 2, 4, 8, 8])
    dim = rng.choice([64, 128, 128, 128, 256, 16 * rng.randint(2, 16)])
    page = rng.choice([16, 32, 48, 64, 128])
    fmt = rng.choice(["int8", "fp8"])
    if kind == "append":
        new = rng.choice([1, 1, _log_int(rng, 2, 8), _log_int(rng, 9, 4096)])
        seqs = _log_int(rng, 1, max(1, min(64, 16384 // new)))
        length = _log_int(rng, new, max(new, min(8192, (1 << 20) // seqs)))
        return dict(kind=kind, seqs=seqs, new=new, len=length, ragged=rng.random() < 0.5, heads=heads, dim=dim, page=page,
                    fmt=fmt, type=typ, rot=rng.choice([0, dim, dim // 2]), interleaved=rng.random() < 0.5)
    qh = heads * rng.choice([1, 2, 4, 4, 5, 8])
    qh = qh if qh <= 40 else heads
    new = rng.choice([1, 1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 4096)])
    if new <= 16:
        seqs = _log_int(rng, 1, 64)
        length = max(new, _log_int(rng, 1, max(64, min(131071, (1 << 17) // seqs))))
    else:
        seqs = _log_int(rng, 1, max(1, min(6, 8192 // new)))
        length = new + rng.choice([0, _log_int(rng, 1, 4096)])
        while seqs * new * length * qh * dim * (1 if typ == "bf16" else 3) > 2e11:
            new, length = max(1, new // 2), max(1, length // 2)
    return dict(kind=kind, seqs=seqs, new=new, len=length, ragged=rng.random() < 0.5, qh=qh, heads=heads, dim=dim, page=page,
                fmt=fmt, type=typ, causal=rng.random() < 0.8, window=rng.choice([0, 0, 0, _log_int(rng, 1, 4096)]))


# ---- inputs, from the seed alone ---------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _page_bytes(page, heads, dim):
    return -(-(2 * page * heads * dim + page * heads // 2) // 128) * 128


def _lengths(case):
    """(new rows, tokens with them) of every sequence; the same for every seed."""
    g = torch.Generator()
    g.manual_seed(1000 * case["len"] + case["new"])
    out = []
    for _ in range(case["seqs"]):
        new, length = case["new"], case["len"]
        if case["ragged"]:
            if new > 16:
                new = max(1, int(new * (0.1 + 0.9 * torch.rand((), generator=g).item())))
            length = max(new, int(length * (0.1 + 0.9 * torch.rand((), generator=g).item())))
        out.append((new, length))
    return out


def _power(amax):
    """The least power of two that amax is at most 448 times of."""
    mantissa, exponent = torch.frexp(amax.clamp(min=2.0 ** -100))      # amax = mantissa 2^exponent, mantissa in [1/2, 1)
    return ((exponent - torch.where(mantissa <= 0.875, 9, 8) + 127) << 23).to(torch.int32).view(torch.float32)


def _coded(x, fmt):
    """Blocks x [.., n] -> codes as bytes [.., n] and scales [..]: for the inputs alone."""
    amax = x.abs().amax(dim=-1)
    if fmt == "int8":
        scale = amax / 127.0
        return torch.round(x / scale[..., None]).to(torch.int8).view(torch.uint8), scale
    scale = _power(amax)
    return (x / scale[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _store(case, lengths, g):
    """A cache whose pages lie in no order: bytes of every page, the pages of every sequence, its tokens.
    Keys have a few large channels and values tails, as activations do."""
    heads, dim, page = case["heads"], case["dim"], case["page"]
    per_seq = [-(-length // page) for _, length in lengths]
    width = max(per_seq) + 1
    pages = sum(per_seq) + 3
    store = torch.zeros((pages, _page_bytes(page, heads, dim)), dtype=torch.uint8, device=DEV)
    channel = torch.randn((heads, dim), device=DEV, generator=g).mul(0.7).exp()
    blocks, size = page // BLOCK, heads * page * dim
    step = max(1, (1 << 26) // size)
    for a in range(0, pages, step):
        n = min(step, pages - a)
        k = torch.randn((n, heads, blocks, BLOCK, dim), device=DEV, generator=g) * channel[:, None, None, :]
        v = torch.randn((n, heads, blocks, dim, BLOCK), device=DEV, generator=g)
        v = v * (1 + 0.3 * v.abs())
        kc, ks = _coded(k.reshape(n, heads, blocks, -1), case["fmt"])
        vc, vs = _coded(v.reshape(n, heads, blocks, -1), case["fmt"])
        store[a:a + n, :size] = kc.reshape(n, -1)
        store[a:a + n, size:2 * size] = vc.reshape(n, -1)
        scales = torch.cat([ks.reshape(n, -1), vs.reshape(n, -1)], dim=1).contiguous()
        store[a:a + n, 2 * size:2 * size + 8 * heads * blocks] = scales.view(torch.uint8)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, n in enumerate(per_seq):
        table[s, :n] = order[at:at + n]
        at += n
    lens = torch.tensor([length for _, length in lengths], dtype=torch.int32, device=DEV)
    return dict(store=store, table=table, lens=lens)


def _starts(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _angles(rot, positions):
    """cos, sin [positions][rot / 2] as fp32 from 64-bit angles: the table a program builds once."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    t = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.stack([t.cos(), t.sin()], dim=2).float().contiguous()


def _inputs(case, seed):
    g = _gen(seed)
    kind, typ = case["kind"], TYPES[case["type"]]
    if kind == "rotary":
        x = torch.randn((case["rows"], case["heads"], case["dim"]), device=DEV, generator=g).to(typ)
        first = torch.randint(0, case["max_pos"] - min(case["rows"], 1024), (), device=DEV, generator=g)
        pos = (first + torch.arange(case["rows"], device=DEV) % 1024).to(torch.int32)     # sequences of up to 1024
        return dict(x=x, pos=pos, table=_angles(case["rot"], case["max_pos"]))
    if kind == "verify":
        b, k, v = case["seqs"], case["drafts"], case["vocab"]
        z = torch.randn((b, k + 1, v), device=DEV, generator=g) * 3.0
        p = torch.softmax(z, dim=2)
        q = torch.softmax(z[:, :k] + torch.randn((b, k, v), device=DEV, generator=g) * 0.4, dim=2)
        gumbel = -torch.log(-torch.log(torch.rand((b, k, v), device=DEV, generator=g).clamp_(1e-7, 1 - 1e-7)))
        drafts = (q.log() + gumbel).argmax(dim=2).to(torch.int32)
        u = torch.rand((b, k + 1), device=DEV, generator=g)
        return dict(p=p.to(typ), q=q.to(typ) if case["draft_probs"] else None, drafts=drafts, u=u)
    lengths = _lengths(case)
    s = _store(case, lengths, g)
    counts = [n for n, _ in lengths]
    s["lengths"], s["rows"] = lengths, sum(counts)
    s["starts"] = torch.tensor(_starts(counts), dtype=torch.int32, device=DEV)
    if kind == "attn":
        s["q"] = (torch.randn((s["rows"], case["qh"], case["dim"]), device=DEV, generator=g) * 1.5).to(typ)
        return s
    shape = (s["rows"], case["heads"], case["dim"])
    s["k"] = (torch.randn(shape, device=DEV, generator=g) * 1.5).to(typ)
    s["v"] = torch.randn(shape, device=DEV, generator=g).to(typ)
    s["angles"] = _angles(case["rot"], max(length for _, length in lengths)) if case["rot"] else None
    # what is read back: the new tokens and those before them that can share their first one's scale
    s["back"] = [n + BLOCK - 1 for n in counts]
    s["back_starts"] = torch.tensor(_starts(s["back"]), dtype=torch.int32, device=DEV)
    return s


# ---- what a program holds before the call, and the call ------------------------------------------------

def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    kind = case["kind"]
    if kind == "append":
        s["touched"] = _touched(s["lengths"])
    if not own:
        return s
    import paper_2005_09904_amd as biq

    if kind == "rotary":
        s["y"] = torch.empty_like(s["x"])
        s["call"] = biq.PreparedRotary(s["x"], s["y"], s["pos"], s["table"], interleaved=case["interleaved"],
                                       inverse=case["inverse"])
        return s
    if kind == "verify":
        b, k = case["seqs"], case["drafts"]
        s["tokens"] = torch.empty((b, k + 1), dtype=torch.int32, device=DEV)
        s["accepted"] = torch.empty(b, dtype=torch.int32, device=DEV)
        s["ws"] = torch.empty(max(16, biq.biq_verify_workspace_bytes(b, case["vocab"])), dtype=torch.uint8, device=DEV)
        s["call"] = biq.PreparedVerify(s["p"], s["q"], s["drafts"], s["u"], s["tokens"], s["accepted"], workspace=s["ws"])
        return s
    cache = biq.KvCache(s["store"], s["table"], s["lens"], case["page"], case["heads"], case["dim"], case["fmt"])
    new = max(n for n, _ in s["lengths"])
    if kind == "attn":
        longest = max(length for _, length in s["lengths"])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((s["rows"], case["qh"]), device=DEV)
        how = dict(scale=case["dim"] ** -0.5, starts=s["starts"], max_rows=new, max_len=longest, causal=case["causal"],
                   window=case["window"])
        s["ws"] = torch.empty(max(16, biq.biq_attention_workspace_bytes(cache, s["q"], **how)), dtype=torch.uint8, device=DEV)
        s["call"] = biq.PreparedAttention(cache, s["q"], s["out"], lse=s["lse"], workspace=s["ws"], **how)
        return s
    rows = sum(s["back"])
    s["out_k"] = torch.empty((rows, case["heads"], case["dim"]), device=DEV)
    s["out_v"] = torch.empty_like(s["out_k"])
    s["call"] = biq.PreparedAppend(cache, s["k"], s["v"], starts=s["starts"], max_rows=new, angles=s["angles"],
                                   interleaved=case["interleaved"])
    s["read"] = biq.PreparedRead(cache, s["out_k"], s["out_v"], starts=s["back_starts"], max_rows=max(s["back"]))
    return s


def run(state):
    c = state["case"]
    kind = c["kind"]
    if not own:
        return {"attn": _plain_attention, "append": _plain_append, "rotary": _plain_rotary, "verify": _plain_verify}[kind](state)
    state["call"]()
    if kind == "rotary":
        return state["y"]
    if kind == "verify":
        return [state["tokens"], state["accepted"]]
    if kind == "attn":
        return [state["out"], state["lse"]]
    state["read"]()
    return [state["out_k"], state["out_v"]]


def _visible(case, new, length):
    """Query-token pairs of one sequence."""
    total = 0
    if not case["causal"] and not case["window"]:
        return new * length
    first = length - new
    w = case["window"] or length
    if not case["causal"]:
        return sum(length - max(0, first + i - w + 1) for i in range(new))
    for i in range(new):
        total += min(first + i + 1, w)
    return total


def work(case):
    """Bytes: every input and output once (the cache's visible tokens with their scales).  Operations: products and sums of
    both matrix products; of a rotation; none that are counted for a verification."""
    kind, size = case["kind"], 4 if case["type"] == "fp32" else 2
    if kind == "rotary":
        n = case["rows"] * case["heads"]
        return dict(bytes=2 * n * case["dim"] * size + min(case["rows"], 1024) * case["rot"] * 4 + 4 * case["rows"],
                    flops=3 * n * case["rot"])
    if kind == "verify":
        rows = 2 if case["draft_probs"] else 1
        return dict(bytes=case["seqs"] * (rows * case["vocab"] * size + 4 * (3 * case["drafts"] + 3)), flops=0)
    lengths = _lengths(case)
    heads, dim = case["heads"], case["dim"]
    token = heads * (2 * dim + 8 / BLOCK)
    if kind == "append":
        rows = sum(n for n, _ in lengths)
        back = sum(n + BLOCK - 1 for n, _ in lengths)
        return dict(bytes=int(2 * rows * heads * dim * size + rows * token + 2 * back * heads * dim * 4),
                    flops=3 * rows * heads * case["rot"])
    seen = sum(min(length, case["window"] + n - 1) if case["window"] else length for n, length in lengths)
    rows = sum(n for n, _ in lengths)
    return dict(bytes=int(seen * token + rows * case["qh"] * (2 * dim * size + 4)),
                flops=4 * case["qh"] * dim * sum(_visible(case, n, length) for n, length in lengths))


# ---- the plain forms ---------------------------------------------------------------------------------

def _values(case, pages):
    """Pages [n, bytes] -> keys and values [tokens, heads, dim] in 32 bits."""
    heads, dim, page = case["heads"], case["dim"], case["page"]
    n, blocks, size = pages.shape[0], page // BLOCK, heads * page * dim
    code = torch.int8 if case["fmt"] == "int8" else torch.float8_e4m3fn
    scales = pages[:, 2 * size:2 * size + 8 * heads * blocks].contiguous().view(torch.float32).reshape(n, 2, heads, blocks, 1, 1)
    k = pages[:, :size].contiguous().view(code).float().reshape(n, heads, blocks, BLOCK, dim) * scales[:, 0]
    v = pages[:, size:2 * size].contiguous().view(code).float().reshape(n, heads, blocks, dim, BLOCK) * scales[:, 1]
    return (k.permute(0, 2, 3, 1, 4).reshape(n * page, heads, dim), v.permute(0, 2, 4, 1, 3).reshape(n * page, heads, dim))


def _plain_attention(state):
    c = state["case"]
    qh, heads, dim, typ = c["qh"], c["heads"], c["dim"], TYPES[c["type"]]
    outs, lses, at = [], [], 0
    for s, (new, length) in enumerate(state["lengths"]):
        pages = state["table"][s, :-(-length // c["page"])].long()
        k, v = _values(c, state["store"][pages])
        k, v = k[:length].permute(1, 2, 0).contiguous(), v[:length].permute(1, 0, 2).contiguous()
        q = state["q"][at:at + new].float().permute(1, 0, 2).reshape(heads, qh // heads * new, dim)
        scores = torch.matmul(q, k).reshape(heads, qh // heads, new, length) * dim ** -0.5
        if c["causal"] or c["window"]:
            pos = torch.arange(length - new, length, device=DEV)[:, None]
            t = torch.arange(length, device=DEV)[None, :]
            hidden = torch.zeros((new, length), dtype=torch.bool, device=DEV)
            if c["causal"]:
                hidden |= t > pos
            if c["window"]:
                hidden |= t <= pos - c["window"]
            scores.masked_fill_(hidden, float("-inf"))
        top = scores.amax(dim=3, keepdim=True)
        e = torch.exp_(scores.sub_(top))
        total = e.sum(dim=3, keepdim=True)
        out = torch.matmul(e.reshape(heads, -1, length), v).reshape(heads, -1, new, dim) / total
        outs.append(out.reshape(qh, new, dim).permute(1, 0, 2))
        lses.append((top + torch.log(total)).reshape(qh, new).t())
        at += new
    return [torch.cat(outs).to(typ), torch.cat(lses).contiguous()]


def _rotated(x, cos, sin, rot, interleaved):
    """x [rows, heads, dim] in 32 bits, cos and sin [rows, rot / 2]."""
    c, s = cos[:, None, :], sin[:, None, :]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * s, a * s + b * c
    return y


def _plain_rotary(state):
    c = state["case"]
    t = state["table"][state["pos"].long()]
    sin = -t[..., 1] if c["inverse"] else t[..., 1]
    return _rotated(state["x"].float(), t[..., 0], sin, c["rot"], c["interleaved"]).to(state["x"].dtype)


def _touched(lengths):
    """(sequence, block) pairs that a call changes, and the rows of the input in each block."""
    seq, block, row = [], [], []
    at = 0
    for s, (new, length) in enumerate(lengths):
        first = length - new
        for b in range(first // BLOCK, -(-length // BLOCK)):
            seq.append(s)
            block.append(b)
            row.append([at + t - first if first <= t < length else -1 for t in range(b * BLOCK, (b + 1) * BLOCK)])
        at += new
    to = lambda a: torch.tensor(a, dtype=torch.int64, device=DEV)
    first = [lengths[s][1] - lengths[s][0] for s in seq]
    return dict(seq=to(seq), block=to(block), row=to(row), old=to([max(0, min(BLOCK, f - b * BLOCK)) for f, b in zip(first, block)]))


def _plain_codes(x, old_codes, old_scale, fmt, is_new, is_old):
    """New values x, codes before (as numbers) and their scale, per block [.., n] -> codes as numbers, scale."""
    amax = torch.where(is_new, x, 0.0).abs().amax(dim=(-2, -1))
    if fmt == "int8":
        scale = amax / 127.0
    else:
        scale = _power(amax)
    scale = torch.where(amax < 2.0 ** -100, torch.zeros_like(scale), scale)
    scale = torch.maximum(scale, old_scale)
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))[..., None, None]
    keep = torch.where(scale > 0, old_scale / scale, torch.zeros_like(scale))[..., None, None]
    wanted = torch.where(is_new, x * inv, torch.where(is_old, old_codes * keep, 0.0))
    if fmt == "int8":
        return torch.round(wanted).clamp(-127, 127), scale
    return wanted.to(torch.float8_e4m3fn).float(), scale


def _plain_append(state):
    c, t = state["case"], state["touched"]
    heads, dim, page, store = c["heads"], c["dim"], c["page"], state["store"]
    k, v = state["k"].float(), state["v"].float()
    if c["rot"]:
        counts = torch.diff(state["starts"])
        last = torch.repeat_interleave(state["lens"] - state["starts"][1:], counts.long(), output_size=state["rows"])
        pos = (torch.arange(state["rows"], device=DEV) + last).long()
        a = state["angles"][pos]
        k = _rotated(k, a[..., 0], a[..., 1], c["rot"], c["interleaved"])
    blocks, size = page // BLOCK, heads * page * dim
    pg = state["table"][t["seq"], t["block"] * BLOCK // page].long()
    sub = t["block"] % blocks
    n = pg.shape[0]
    code = torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn
    flat = store.view(-1)
    at = (pg * store.shape[1])[:, None] + (torch.arange(heads, device=DEV) * blocks)[None, :] * (BLOCK * dim) + (sub * (BLOCK * dim))[:, None]
    at = at[..., None] + torch.arange(BLOCK * dim, device=DEV)                               # bytes of a block and head
    scale_at = (pg * (store.shape[1] // 4))[:, None] + size // 2 + (torch.arange(heads, device=DEV) * blocks)[None, :] + sub[:, None]
    floats = flat.view(torch.float32)
    is_new = (t["row"] >= 0)
    is_old = torch.arange(BLOCK, device=DEV)[None, :] < t["old"][:, None]
    for which, x in enumerate((k, v)):
        x = x[t["row"].clamp(min=0)].permute(0, 2, 1, 3)                                  # [n, heads, 16, dim]
        x = x if which == 0 else x.transpose(2, 3)
        shape = (n, 1, BLOCK, 1) if which == 0 else (n, 1, 1, BLOCK)
        here, there = at + which * size, scale_at + which * heads * blocks
        old = flat[here].view(code).float().reshape(x.shape)
        old_scale = torch.where((t["old"] > 0)[:, None], floats[there], 0.0)
        codes, scale = _plain_codes(x, old, old_scale, c["fmt"], is_new.reshape(shape), is_old.reshape(shape))
        flat[here] = codes.to(code).view(torch.uint8).reshape(n, heads, -1)
        floats[there] = scale
    # read back
    outs = ([], [])
    for s, (new, length) in enumerate(state["lengths"]):
        first = length - new - (BLOCK - 1)
        p0 = max(0, first) // page
        vals = _values(c, store[state["table"][s, p0:-(-length // page)].long()])
        for out, val in zip(outs, vals):
            got = val[max(0, first) - p0 * page:length - p0 * page]
            out.append(got if first >= 0 else torch.cat([torch.zeros((-first, heads, dim), device=DEV), got]))
    return [torch.cat(outs[0]), torch.cat(outs[1])]


def _plain_verify(state):
    p, q, drafts, u = state["p"].float(), state["q"], state["drafts"].long(), state["u"]
    b, k = drafts.shape
    pt = p[:, :k].gather(2, drafts[..., None])[..., 0]
    if q is None:
        ok = u[:, :k] < pt
    else:
        ok = u[:, :k] * q.float().gather(2, drafts[..., None])[..., 0] < pt
    accepted = ok.long().cumprod(dim=1).sum(dim=1)
    rows = torch.arange(b, device=DEV)
    at = accepted.clamp(max=k - 1)
    target = p[rows, accepted]
    if q is None:
        draft = torch.zeros_like(target)
        draft[rows, drafts[rows, at]] = 1.0
    else:
        draft = q[rows, at].float()
    rest = torch.where((accepted < k)[:, None], target - draft, target)

    def weights(r):
        r = torch.where(r > 0, r, 0.0).clamp(max=1.0)
        return (r * 2.0 ** 40).long()

    w = weights(rest)
    w = torch.where((w.sum(dim=1) == 0)[:, None], weights(target), w)
    sums = w.cumsum(dim=1)
    total = sums[:, -1]
    x = (u[:, k] * 2.0 ** 31).long()
    goal = x * (total >> 32) * 2 + (x * (total & 0xffffffff) >> 31)
    token = (sums <= goal[:, None]).sum(dim=1)
    token = torch.where(total > 0, token, -1)
    tokens = torch.full((b, k + 1), -1, dtype=torch.int64, device=DEV)
    tokens[:, :k] = torch.where(torch.arange(k, device=DEV) < accepted[:, None], drafts, -1)
    tokens.scatter_(1, accepted[:, None], token[:, None])
    return [tokens.int(), accepted.int()]


# ---- the same in 64 bits ---------------------------------------------------------------------------------

def _decode64(fmt, raw):
    """The numbers that code bytes stand for."""
    i = torch.arange(256, device=DEV, dtype=torch.float64)
    if fmt == "int8":
        return torch.where(i < 128, i, i - 256)[raw.long()]
    exponent, fraction = (i // 8) % 16, i % 8
    value = torch.where(exponent == 0, fraction * 2.0 ** -9, (1 + fraction / 8) * torch.pow(2.0, exponent - 7))
    value[[127, 255]] = float("nan")
    return torch.where(i < 128, value, -value)[raw.long()]


def _tokens64(case, s, seq, head):
    """Keys and values [length, dim] of one sequence and head."""
    heads, dim, page = case["heads"], case["dim"], case["page"]
    length, blocks = s["lengths"][seq][1], page // BLOCK
    pages = s["store"][s["table"][seq, :-(-length // page)].long()]
    bytes_ = blocks * BLOCK * dim
    k = _decode64(case["fmt"], pages[:, head * bytes_:(head + 1) * bytes_]).reshape(-1, BLOCK, dim)
    v = _decode64(case["fmt"], pages[:, (heads + head) * bytes_:(heads + head + 1) * bytes_]).reshape(-1, dim, BLOCK)
    floats = pages.view(torch.float32)[:, 2 * heads * bytes_ // 4:].double()
    ks = floats[:, head * blocks:(head + 1) * blocks].reshape(-1)
    vs = floats[:, (heads + head) * blocks:(heads + head + 1) * blocks].reshape(-1)
    k, v = k * ks[:, None, None], (v * vs[:, None, None]).transpose(1, 2)
    return k.reshape(-1, dim)[:length], v.reshape(-1, dim)[:length]


def _exact_attention(case, s):
    group = case["qh"] // case["heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], float("-inf"), dtype=torch.float64, device=DEV)
    at = 0
    for seq, (new, length) in enumerate(s["lengths"]):
        for head in range(case["heads"]):
            k, v = _tokens64(case, s, seq, head)
            for h in range(head * group, (head + 1) * group):
                z = s["q"][at:at + new, h].double() @ k.t().contiguous() / math.sqrt(case["dim"])
                lag = torch.arange(length - new, length, device=DEV)[:, None] - torch.arange(length, device=DEV)
                if case["causal"]:
                    z[lag < 0] = float("-inf")
                if case["window"]:
                    z[lag >= case["window"]] = float("-inf")
                lse[at:at + new, h] = torch.logsumexp(z, dim=1)
                out[at:at + new, h] = torch.exp(z - lse[at:at + new, h, None]) @ v
        at += new
    return [out, lse]


def _exact_rotation(x, t, rot, interleaved, inverse):
    """x [rows, heads, dim] in 64 bits as complex numbers, turned by the table's angles [rows, rot / 2, 2]."""
    turn = torch.complex(t[..., 0].double(), -t[..., 1].double() if inverse else t[..., 1].double())[:, None, :]
    pair = x[..., :rot].reshape(*x.shape[:2], rot // 2, 2) if interleaved else x[..., :rot].reshape(*x.shape[:2], 2, rot // 2).transpose(2, 3)
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
    z = z if interleaved else z.transpose(2, 3)
    return torch.cat([z.reshape(*x.shape[:2], rot), x[..., rot:]], dim=2)


def _round64(x, fmt):
    if fmt == "int8":
        return x.round().clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.clamp((x / step).round() * step, -448, 448)


def _exact_append(case, s):
    k, v = s["k"].double(), s["v"].double()
    top = 127.0 if case["fmt"] == "int8" else 448.0
    outs = ([], [])
    at = 0
    for seq, (new, length) in enumerate(s["lengths"]):
        first = length - new
        kn = k[at:at + new]
        if case["rot"]:
            kn = _exact_rotation(kn, s["angles"][first:length], case["rot"], case["interleaved"], False)
        base = max(0, first - (BLOCK - 1)) // BLOCK * BLOCK
        end = -(-length // BLOCK) * BLOCK
        before = [torch.stack([_tokens64_block(case, s, seq, h, base, end, w) for h in range(case["heads"])], dim=1) for w in (0, 1)]
        for w, x in enumerate((kn, v[at:at + new])):
            codes, scale = before[w][..., :-1], before[w][..., -1]                 # [tokens, heads, dim], [tokens, heads]
            val = codes * scale[..., None]
            b0 = first // BLOCK * BLOCK
            pad = torch.zeros((end - b0, case["heads"], case["dim"]), dtype=torch.float64, device=DEV)
            pad[first - b0:first - b0 + new] = x
            blk = pad.reshape(-1, BLOCK, case["heads"], case["dim"])
            need = blk.abs().amax(dim=(1, 3)) / top
            if case["fmt"] == "fp8":
                need = torch.exp2(torch.ceil(torch.log2(need)))
            held = torch.zeros_like(need)
            if first % BLOCK:
                held[0] = scale[b0 - base]
            now = torch.maximum(need, held)[:, None, :, None]
            kept = torch.zeros_like(pad)
            kept[:first - b0] = val[b0 - base:first - base]
            val[b0 - base:] = (_round64((blk + kept.reshape(blk.shape)) / now, case["fmt"]) * now).reshape(pad.shape)
            lead = first - (BLOCK - 1)
            got = val[max(0, lead) - base:length - base]
            outs[w].append(torch.cat([torch.zeros((max(0, -lead), case["heads"], case["dim"]), dtype=torch.float64, device=DEV), got]))
        at += new
    return [torch.cat(outs[0]), torch.cat(outs[1])]


def _tokens64_block(case, s, seq, head, base, end, which):
    """Codes [tokens, dim] of positions base..end of one sequence and head, each with its scale after them."""
    heads, dim, page = case["heads"], case["dim"], case["page"]
    block = torch.arange(base // BLOCK, end // BLOCK, device=DEV)
    pages = s["store"][s["table"][seq, (block * BLOCK // page)].long()]
    sub = (block % (page // BLOCK)) + (which * heads + head) * (page // BLOCK)
    raw = pages.gather(1, (sub * BLOCK * dim)[:, None] + torch.arange(BLOCK * dim, device=DEV))
    code = _decode64(case["fmt"], raw)
    code = code.reshape(-1, BLOCK, dim) if which == 0 else code.reshape(-1, dim, BLOCK).transpose(1, 2)
    scale = pages.view(torch.float32).gather(1, (2 * heads * page * dim // 4 + sub)[:, None])[:, :, None].double()
    return torch.cat([code, scale.expand(-1, BLOCK, 1)], dim=2).reshape(-1, dim + 1)


def exact(case, seed):
    kind = case["kind"]
    if kind == "verify":
        return None                       # whole numbers: equal to the plain form's or wrong
    s = _inputs(case, seed)
    if kind == "rotary":
        return _exact_rotation(s["x"].double(), s["table"][s["pos"].long()], case["rot"], case["interleaved"], case["inverse"])
    return _exact_attention(case, s) if kind == "attn" else _exact_append(case, s)
