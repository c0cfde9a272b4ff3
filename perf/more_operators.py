"""The end of a decoder step and attention of a batch with a common prefix, as cases that can be timed and checked: the
norm with the residual's addition, products with 4-bit weights, penalties and masks on logits, attention that reads a
shared prefix once.

A case is one call of a public entry point.  `run` makes it, or, where `own` is false, computes the same in elementary
torch operations in 32 bits.  Sizes are generic or those of the benchmark's layers.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8, "fp8": torch.float8_e4m3fn}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2, "int8": 1, "fp8": 1}
BLOCK = 16                                    # tokens of the cache that share a scale
EPS = 1e-6


def listed():
    return [
        # -- norm ---------------------------------------------------------------------------------------
        # before a projection of a single token: launch and two dependent steps
        dict(name="norm_token", kind="norm", rows=1, n=4096, type="fp32", y="fp32", residual=True, weight_add=0.0, codes="", group=0),
        # a batch with its drafted tokens, whose codes the 4-bit products take; an odd width
        dict(name="norm_codes_b80", kind="norm", rows=80, n=5003, type="bf16", y="", residual=True, weight_add=0.0, codes="int8", group=128),
        # prompts: memory
        dict(name="norm_prompt", kind="norm", rows=8192, n=4096, type="bf16", y="bf16", residual=True, weight_add=1.0, codes="", group=0),
        # -- products with 4-bit weights ----------------------------------------------------------------
        # a square layer and one vector
        dict(name="gemm4_token", kind="gemm4", m=4096, n=4096, batch=1, group=128, x="fp32", x_group=0, y="fp32"),
        # the output head of a single sequence
        dict(name="gemm4_head", kind="gemm4", m=32000, n=4096, batch=1, group=64, x="bf16", x_group=0, y="fp32"),
        # drafted tokens over the wide layer, inputs in 8 bits as the norm gives them
        dict(name="gemm4_drafts_codes", kind="gemm4", m=16384, n=4096, batch=5, group=128, x="int8", x_group=128, y="bf16"),
        # a serving batch over long rows
        dict(name="gemm4_b48", kind="gemm4", m=4096, n=16384, batch=48, group=32, x="fp32", x_group=0, y="fp32"),
        # -- logits -------------------------------------------------------------------------------------
        # one sequence's next token
        dict(name="logits_b1", kind="logits", seqs=1, rows=1, vocab=32000, type="fp32", out="fp32", history=300, bias=0, mask=False,
             probabilities=True),
        # a batch with four drafted tokens each, long histories, a grammar
        dict(name="logits_drafts_b32", kind="logits", seqs=32, rows=5, vocab=120011, type="bf16", out="fp32", history=4000, bias=50,
             mask=True, probabilities=True),
        # -- attention with a common prefix -------------------------------------------------------------
        # a few short answers to one instruction
        dict(name="shared_short", kind="shared", seqs=4, new=1, shared=512, len=100, qh=8, heads=8, dim=64, page=16, fmt="int8",
             type="fp32", causal=True, window=0),
        # a serving batch behind one long instruction
        dict(name="shared_token_b32", kind="shared", seqs=32, new=1, shared=8192, len=1000, qh=32, heads=8, dim=128, page=64,
             fmt="int8", type="bf16", causal=True, window=0),
        # many answers drawn from one document, drafted tokens to verify
        dict(name="shared_drafts_b24", kind="shared", seqs=24, new=5, shared=32768, len=600, qh=32, heads=8, dim=128, page=128,
             fmt="fp8", type="fp32", causal=True, window=0),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm of [lo, hi], odd values among them."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.3 and v >= 64:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["norm", "norm", "gemm4", "gemm4", "gemm4", "logits", "logits", "shared", "shared", "shared"])
    typ = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if kind == "norm":
        n = rng.choice([_log_int(rng, 64, 16384), 64 * rng.randint(1, 128)])
        codes = rng.choice(["", "", "int8", "fp8"])
        rows = _log_int(rng, 1, max(1, min(8192, (1 << (22 if codes else 25)) // n)))
        return dict(kind=kind, rows=rows, n=n, type=typ, y=rng.choice([typ, "fp32"]) if not codes or rng.random() < 0.3 else "",
                    residual=rng.random() < 0.8, weight_add=rng.choice([0.0, 0.0, 1.0]), codes=codes,
                    group=rng.choice([0, 32, 64, 128, 128]) if codes else 0)
    if kind == "gemm4":
        m, n = _log_int(rng, 64, 32000), _log_int(rng, 64, 16384)
        while m * n > 1.3e8:
            m, n = (m // 2 + 1, n) if rng.random() < 0.5 else (m, n // 2 + 1)
        batch = rng.choice([1, 1, _log_int(rng, 1, 8), _log_int(rng, 2, 64)])
        batch = max(1, min(batch, int(3.2e9 / (m * n))))
        x = rng.choice([typ, typ, "int8", "fp8"])
        return dict(kind=kind, m=m, n=n, batch=batch, group=rng.choice([32, 64, 128, 128]), x=x,
                    x_group=rng.choice([0, 128, 128, 64, 32]) if x in ("int8", "fp8") else 0, y=rng.choice([typ, "fp32"]))
    if kind == "logits":
        seqs = _log_int(rng, 1, 64)
        rows = rng.choice([1, 1, rng.randint(2, 8)])
        vocab = _log_int(rng, 1000, max(1000, min(131072, int(1.9e7 / (seqs * rows)))))
        return dict(kind=kind, seqs=seqs, rows=rows, vocab=vocab, type=typ, out=rng.choice([typ, "fp32", "fp32"]),
                    history=rng.choice([0, _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)]), bias=rng.choice([0, _log_int(rng, 1, 300)]),
                    mask=rng.random() < 0.5, probabilities=rng.random() < 0.7)
    heads = rng.choice([1, 2, 4, 8, 8])
    qh = heads * rng.choice([1, 2, 4, 4, 5])
    dim = rng.choice([64, 128, 128, 128, 256, 16 * rng.randint(2, 16)])
    page = rng.choice([16, 32, 48, 64, 128])
    new = rng.choice([1, 1, 1, _log_int(rng, 2, 8), _log_int(rng, 9, 128)])
    seqs = _log_int(rng, 1, max(1, min(64, 384 // new)))
    shared = page * max(1, _log_int(rng, 64, max(64, min(32768, int(1.5e10 / (seqs * new * qh * dim))))) // page)
    length = max(new, _log_int(rng, 1, max(16, min(4096, (1 << 16) // seqs))))
    return dict(kind=kind, seqs=seqs, new=new, shared=shared, len=length, qh=qh, heads=heads, dim=dim, page=page,
                fmt=rng.choice(["int8", "fp8"]), type=typ, causal=rng.random() < 0.8, window=rng.choice([0, 0, 0, _log_int(rng, 64, 8192)]))


# ---- inputs, from the seed alone ---------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _groups(n, group):
    return 1 if group == 0 else -(-n // group)


def _power(amax):
    """The least power of two that amax is at most 448 times of."""
    mantissa, exponent = torch.frexp(amax.clamp(min=2.0 ** -100))      # amax = mantissa 2^exponent, mantissa in [1/2, 1)
    return ((exponent - torch.where(mantissa <= 0.875, 9, 8) + 127) << 23).to(torch.int32).view(torch.float32)


def _coded(x, fmt):
    """Blocks x [.., n] -> codes and scales [..]: for the inputs alone."""
    amax = x.abs().amax(dim=-1)
    scale = amax / 127.0 if fmt == "int8" else _power(amax)
    y = x / scale[..., None]
    return (torch.round(y).to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)), scale


def _grouped(x, n, group):
    """[rows, n] -> [rows, groups, group], zeros behind the last element."""
    size = n if group == 0 else group
    return torch.nn.functional.pad(x, (0, _groups(n, group) * size - n)).reshape(x.shape[0], -1, size)


def _norm_inputs(case, g):
    rows, n, typ = case["rows"], case["n"], TYPES[case["type"]]
    channel = torch.randn(n, device=DEV, generator=g).mul(0.5).exp()                    # a few large channels
    x = (torch.randn((rows, n), device=DEV, generator=g) * channel * 0.7).to(typ)
    residual = (torch.randn((rows, n), device=DEV, generator=g) * channel * 3).to(typ) if case["residual"] else None
    weight = torch.randn(n, device=DEV, generator=g) * 0.3 + 1.0 - case["weight_add"]
    return dict(x=x, residual=residual, weight=weight)


def _gemm4_inputs(case, g):
    m, n, b, group = case["m"], case["n"], case["batch"], case["group"]
    codes = (torch.randn((m, n), device=DEV, generator=g) * 2.6).round_().clamp_(-8, 7).to(torch.int8)
    scales = (torch.rand((m, _groups(n, group)), device=DEV, generator=g) * 0.02 + 0.01).bfloat16()
    x = torch.randn((b, n), device=DEV, generator=g) * torch.randn(n, device=DEV, generator=g).mul(0.5).exp()
    if case["x"] not in ("int8", "fp8"):
        return dict(codes=codes, scales=scales, x=x.to(TYPES[case["x"]]), x_scales=None)
    c, s = _coded(_grouped(x, n, case["x_group"]), case["x"])
    return dict(codes=codes, scales=scales, x=c.reshape(b, -1).view(torch.uint8)[:, :n].contiguous().view(TYPES[case["x"]]), x_scales=s.contiguous())


def _logits_inputs(case, g):
    seqs, rows, vocab = case["seqs"], case["rows"], case["vocab"]
    s = dict(x=(torch.randn((seqs, rows, vocab), device=DEV, generator=g) * 3.0).to(TYPES[case["type"]]))
    rand = lambda *shape: torch.rand(shape, device=DEV, generator=g)
    often = lambda *shape: (rand(*shape) ** 4 * vocab).long().clamp_(max=vocab - 1).int()      # a text repeats its frequent tokens
    if case["history"]:
        s["history"] = often(seqs, case["history"])
        s["lens"] = (case["history"] * (0.2 + 0.8 * rand(seqs))).int().clamp_(min=1)
        s["prompt_lens"] = (s["lens"] * rand(seqs)).int()
        s["drafts"] = often(seqs, rows - 1)
        s["repetition"], s["presence"], s["frequency"] = 1.0 + 0.3 * rand(seqs), 0.5 * rand(seqs), 0.3 * rand(seqs)
    s["temperature"] = 0.5 + rand(seqs)
    if seqs > 2:
        s["temperature"][1] = 0.0                                  # one that takes the likeliest token
    if case["bias"]:
        s["bias_tokens"], s["bias_values"] = often(seqs, case["bias"]), 4.0 * rand(seqs, case["bias"]) - 2.0
    if case["mask"]:
        words = -(-vocab // 32)
        allowed = rand(seqs, rows, words * 32) < rand(seqs, rows, 1)   # grammars that leave many tokens or few
        allowed[..., 0] = True
        bits = (allowed.reshape(seqs, rows, words, 32).long() << torch.arange(32, device=DEV)).sum(dim=3)
        s["mask"] = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()
    return s


def _page_bytes(page, heads, dim):
    return -(-(2 * page * heads * dim + page * heads // 2) // 128) * 128


def _own_lengths(case):
    """Tokens of every sequence behind the prefix; the same for every seed."""
    g = torch.Generator()
    g.manual_seed(1000 * case["len"] + case["new"])
    return [max(case["new"], int(case["len"] * (0.1 + 0.9 * torch.rand((), generator=g).item()))) for _ in range(case["seqs"])]


def _shared_inputs(case, g):
    heads, dim, page, seqs = case["heads"], case["dim"], case["page"], case["seqs"]
    lengths = _own_lengths(case)
    front = case["shared"] // page
    own_pages = [-(-length // page) for length in lengths]
    pages = front + sum(own_pages) + 3
    blocks, size = page // BLOCK, heads * page * dim
    store = torch.zeros((pages, _page_bytes(page, heads, dim)), dtype=torch.uint8, device=DEV)
    channel = torch.randn((heads, dim), device=DEV, generator=g).mul(0.7).exp()
    step = max(1, (1 << 26) // size)
    for a in range(0, pages, step):
        n = min(step, pages - a)
        k = torch.randn((n, heads, blocks, BLOCK, dim), device=DEV, generator=g) * channel[:, None, None, :]
        v = torch.randn((n, heads, blocks, dim, BLOCK), device=DEV, generator=g)
        v = v * (1 + 0.3 * v.abs())
        kc, ks = _coded(k.reshape(n, heads, blocks, -1), case["fmt"])
        vc, vs = _coded(v.reshape(n, heads, blocks, -1), case["fmt"])
        store[a:a + n, :size] = kc.view(torch.uint8).reshape(n, -1)
        store[a:a + n, size:2 * size] = vc.view(torch.uint8).reshape(n, -1)
        scales = torch.cat([ks.reshape(n, -1), vs.reshape(n, -1)], dim=1).contiguous()
        store[a:a + n, 2 * size:2 * size + 8 * heads * blocks] = scales.view(torch.uint8)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((seqs, front + max(own_pages) + 1), -1, dtype=torch.int32, device=DEV)
    table[:, :front] = order[:front]
    at = front
    for s, n in enumerate(own_pages):
        table[s, front:front + n] = order[at:at + n]
        at += n
    lens = torch.tensor([case["shared"] + n for n in lengths], dtype=torch.int32, device=DEV)
    q = (torch.randn((seqs * case["new"], case["qh"], dim), device=DEV, generator=g) * 1.5).to(TYPES[case["type"]])
    return dict(store=store, table=table, lens=lens, q=q, lengths=lengths)


def _inputs(case, seed):
    return {"norm": _norm_inputs, "gemm4": _gemm4_inputs, "logits": _logits_inputs, "shared": _shared_inputs}[case["kind"]](case, _gen(seed))


# ---- what a program holds before the call, and the call ------------------------------------------------

def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    kind = case["kind"]
    if kind == "gemm4":
        # what both sides keep of the weights is 4 bits each
        c = torch.nn.functional.pad(s["codes"], (0, case["n"] % 2)).view(torch.uint8)
        s["nibbles"] = (c[:, 0::2] & 15) | (c[:, 1::2] << 4)
    if own:
        _prepare_own(case, s)
    s.pop("codes", None)
    return s


def _prepare_own(case, s):
    """Outputs, workspaces, weights laid out, and the call with its arguments converted."""
    import paper_2005_09904_amd as biq

    kind = case["kind"]
    space = lambda n: torch.empty(max(16, n), dtype=torch.uint8, device=DEV)
    if kind == "norm":
        rows, n = case["rows"], case["n"]
        s["y"] = torch.empty((rows, n), dtype=TYPES[case["y"]], device=DEV) if case["y"] else None
        s["sum"] = torch.empty_like(s["x"]) if case["residual"] else None
        codes = None
        if case["codes"]:
            # rows of whole groups, so that a scale can be spread over its group
            groups = _groups(n, case["group"])
            s["out_codes"] = torch.zeros((rows, groups, case["group"] or n), dtype=torch.uint8, device=DEV).view(TYPES[case["codes"]])
            s["out_scales"] = torch.empty((rows, groups), device=DEV)
            codes = s["out_codes"].view(rows, -1)[:, :n]
        s["call"] = biq.PreparedNorm(s["x"], s["y"], weight=s["weight"], weight_add=case["weight_add"], residual=s["residual"], sum=s["sum"],
                                     codes=codes, scales=s.get("out_scales"), group=case["group"], eps=EPS)
    elif kind == "gemm4":
        m, n, group = case["m"], case["n"], case["group"]
        s["packed"] = space(biq.biq_packed4_bytes(m, n, group))
        biq.biq_pack4(s["codes"], s["scales"].float(), s["packed"], m, n, group)
        s["y"] = torch.empty((case["batch"], m), dtype=TYPES[case["y"]], device=DEV)
        s["ws"] = space(biq.biq_gemm4_workspace_bytes(s["packed"], s["x"], s["y"], group, x_scales=s["x_scales"], x_group=case["x_group"]))
        s["call"] = biq.PreparedGemm4(s["packed"], s["x"], s["y"], group, x_scales=s["x_scales"], x_group=case["x_group"], workspace=s["ws"])
    elif kind == "logits":
        s["out"] = torch.empty(s["x"].shape, dtype=TYPES[case["out"]], device=DEV)
        how = {k: s.get(k) for k in ("history", "lens", "prompt_lens", "drafts", "repetition", "presence", "frequency", "temperature", "bias_tokens",
                                     "bias_values", "mask")}
        s["ws"] = space(biq.biq_logits_workspace_bytes(case["seqs"], case["rows"], case["vocab"]))
        s["call"] = biq.PreparedLogits(s["x"], s["out"], probabilities=case["probabilities"], workspace=s["ws"], **how)
    else:
        cache = biq.KvCache(s["store"], s["table"], s["lens"], case["page"], case["heads"], case["dim"], case["fmt"])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], device=DEV)
        how = dict(scale=case["dim"] ** -0.5, max_len=case["shared"] + max(s["lengths"]), causal=case["causal"], window=case["window"])
        s["ws"] = space(biq.biq_attention_shared_workspace_bytes(cache, s["q"], case["shared"], **how))
        s["call"] = biq.PreparedSharedAttention(cache, s["q"], s["out"], case["shared"], lse=s["lse"], workspace=s["ws"], **how)


def run(state):
    c = state["case"]
    kind = c["kind"]
    if not own:
        return {"norm": _plain_norm, "gemm4": _plain_gemm4, "logits": _plain_logits, "shared": _plain_shared}[kind](state)
    state["call"]()
    if kind == "norm":
        # codes as what they stand for, which the plain form computes too
        values = None
        if c["codes"]:
            held = state["out_codes"] if c["codes"] == "int8" else state["out_codes"].float()
            values = (held * state["out_scales"][..., None]).view(c["rows"], -1)[:, :c["n"]]
        return [t for t in (state["y"], state["sum"], values) if t is not None]
    if kind == "gemm4":
        return state["y"]
    if kind == "logits":
        return state["out"]
    return [state["out"], state["lse"]]


def work(case):
    """Bytes: every input and output once (of a cache what is seen, with its scales; the prefix once for all).  Operations: products and
    sums of matrix products; of the others those of each element."""
    kind = case["kind"]
    if kind == "norm":
        n = case["rows"] * case["n"]
        size = BYTES[case["type"]]
        out = (BYTES[case["y"]] if case["y"] else 0) + (1 if case["codes"] else 0)
        scales = 4 * case["rows"] * _groups(case["n"], case["group"]) if case["codes"] else 0
        return dict(bytes=n * (size * (3 if case["residual"] else 1) + out) + scales + 4 * case["n"], flops=6 * n)
    if kind == "gemm4":
        m, n, b = case["m"], case["n"], case["batch"]
        xs = 4 * b * _groups(n, case["x_group"]) if case["x"] in ("int8", "fp8") else 0
        return dict(bytes=m * n // 2 + 2 * m * _groups(n, case["group"]) + b * n * BYTES[case["x"]] + xs + b * m * BYTES[case["y"]], flops=2 * m * n * b)
    if kind == "logits":
        rows = case["seqs"] * case["rows"]
        n = rows * case["vocab"]
        return dict(bytes=n * (BYTES[case["type"]] + BYTES[case["out"]]) + (n // 8 if case["mask"] else 0) +
                    case["seqs"] * (4 * case["history"] + 8 * case["bias"] + 24), flops=5 * n)
    token = case["heads"] * (2 * case["dim"] + 8 / BLOCK)
    lengths, new, w = _own_lengths(case), case["new"], case["window"]
    seen = pairs = 0
    front = 0
    for own_len in lengths:
        length = case["shared"] + own_len
        lo = max(0, length - new - w + 1) if w else 0                    # the first token that a row sees
        front = max(front, case["shared"] - lo)
        seen += length - max(lo, case["shared"])
        for i in range(new):
            pos = length - new + i
            pairs += (pos + 1 if case["causal"] else length) - (max(0, pos - w + 1) if w else 0)
    rows = case["seqs"] * new
    return dict(bytes=int((max(front, 0) + seen) * token + rows * case["qh"] * (2 * case["dim"] * BYTES[case["type"]] + 4)),
                flops=4 * case["qh"] * case["dim"] * pairs)


# ---- the plain forms ---------------------------------------------------------------------------------

def _plain_norm(state):
    c = state["case"]
    x, w = state["x"].float(), state["weight"] + c["weight_add"]
    s = x + state["residual"].float() if c["residual"] else x
    r = torch.rsqrt(s.square().mean(dim=1, keepdim=True) + EPS)
    out = []
    if c["y"]:
        out.append((s * r * w).to(TYPES[c["y"]]))
    if c["residual"]:
        out.append(s.to(TYPES[c["type"]]))
    if c["codes"]:
        t = _grouped(s * w, c["n"], c["group"])
        amax = t.abs().amax(dim=2, keepdim=True)
        scale = amax * (1.0 / 127.0) if c["codes"] == "int8" else _power(amax)
        scale = torch.where(amax < 2.0 ** -100, 0.0, scale)
        t = t * torch.where(scale > 0, 1.0 / scale, 0.0)
        t = torch.round(t).clamp(-127, 127) if c["codes"] == "int8" else t.to(torch.float8_e4m3fn).float()
        out.append((t * (scale * r[..., None])).reshape(c["rows"], -1)[:, :c["n"]])
    return out


def _spread(scales, n, group):
    """A scale for each of n elements of the rows."""
    return scales if group == 0 else scales.repeat_interleave(group, dim=1)[:, :n]


def _plain_gemm4(state):
    c = state["case"]
    n = c["n"]
    low, high = state["nibbles"] & 15, state["nibbles"] >> 4
    codes = torch.stack([low, high], dim=2).reshape(c["m"], -1)[:, :n].float()
    w = torch.where(codes > 7, codes - 16, codes) * _spread(state["scales"].float(), n, c["group"])
    x = state["x"].float() if state["x_scales"] is None else state["x"].float() * _spread(state["x_scales"], n, c["x_group"])
    return torch.matmul(x, w.t()).to(TYPES[c["y"]])


def _plain_logits(state):
    c = state["case"]
    seqs, rows, vocab = c["seqs"], c["rows"], c["vocab"]
    z = state["x"].float()
    each = lambda name: state[name][:, None, None]
    if c["history"]:
        t = torch.arange(c["history"], device=DEV)[None, :]
        there, answer = t < state["lens"][:, None], t >= state["prompt_lens"][:, None]
        history = state["history"].long()
        zero = torch.zeros((seqs, vocab), device=DEV)
        prompt = zero.scatter_add(1, history, (there & ~answer).float())
        said = zero.scatter_add(1, history, (there & answer).float())
        # the drafts before a row have been said by then
        more = torch.zeros((seqs, rows, vocab), device=DEV)
        more[:, 1:].scatter_(2, state["drafts"].long()[..., None], 1.0)
        said = said[:, None] + more.cumsum(dim=1)
        seen = (prompt[:, None] + said) > 0
        z = torch.where(seen, torch.where(z > 0, z / each("repetition"), z * each("repetition")), z)
        z = z - said * each("frequency")
        z = torch.where(said > 0, z - each("presence"), z)
    if c["bias"]:
        z = z + torch.zeros((seqs, vocab), device=DEV).scatter_add(1, state["bias_tokens"].long(), state["bias_values"])[:, None]
    hot = each("temperature")
    z = torch.where(hot > 0, z / torch.where(hot > 0, hot, 1.0), z)
    if c["mask"]:
        bits = (state["mask"][..., None] >> torch.arange(32, device=DEV)) & 1
        z = torch.where(bits.reshape(seqs, rows, -1)[..., :vocab] > 0, z, float("-inf"))
    if c["probabilities"]:
        e = torch.exp(z - z.amax(dim=2, keepdim=True))
        p = e / e.sum(dim=2, keepdim=True)
        first = torch.zeros_like(z).scatter_(2, z.argmax(dim=2, keepdim=True), 1.0)
        z = torch.where(hot > 0, p, first)
    return z.to(TYPES[c["out"]])


def _values(case, pages):
    """Pages [.., bytes] -> keys and values [.., tokens, heads, dim] in 32 bits."""
    heads, dim, page = case["heads"], case["dim"], case["page"]
    lead, pages = pages.shape[:-2], pages.reshape(-1, pages.shape[-1])
    n, blocks, size = pages.shape[0], page // BLOCK, heads * page * dim
    code = TYPES[case["fmt"]]
    scales = pages[:, 2 * size:2 * size + 8 * heads * blocks].contiguous().view(torch.float32).reshape(n, 2, heads, blocks, 1, 1)
    k = pages[:, :size].contiguous().view(code).float().reshape(n, heads, blocks, BLOCK, dim) * scales[:, 0]
    v = pages[:, size:2 * size].contiguous().view(code).float().reshape(n, heads, blocks, dim, BLOCK) * scales[:, 1]
    return k.permute(0, 2, 3, 1, 4).reshape(*lead, -1, heads, dim), v.permute(0, 2, 4, 1, 3).reshape(*lead, -1, heads, dim)


def _plain_shared(state):
    c = state["case"]
    seqs, new, heads, dim, qh = c["seqs"], c["new"], c["heads"], c["dim"], c["qh"]
    group, front = qh // heads, c["shared"] // c["page"]
    behind = -(-max(state["lengths"]) // c["page"])
    k0, v0 = _values(c, state["store"][state["table"][0, :front].long()])
    pages = state["table"][:, front:front + behind]
    k1, v1 = _values(c, torch.where((pages >= 0)[..., None], state["store"][pages.clamp(min=0).long()], 0))
    q = state["q"].float().reshape(seqs, new, heads, group, dim).permute(2, 0, 3, 1, 4)                        # [heads, seqs, group, new, dim]
    s0 = torch.matmul(q.reshape(heads, -1, dim), k0.permute(1, 2, 0).contiguous()).reshape(heads, seqs, group, new, -1)
    s1 = torch.matmul(q.reshape(heads, seqs, group * new, dim), k1.permute(2, 0, 3, 1).contiguous()).reshape(heads, seqs, group, new, -1)
    scores = torch.cat([s0, s1], dim=4) * dim ** -0.5
    t = torch.arange(scores.shape[4], device=DEV)
    pos = state["lens"][:, None] - new + torch.arange(new, device=DEV)
    hidden = t >= state["lens"][:, None, None].expand(seqs, new, 1)
    if c["causal"]:
        hidden = hidden | (t > pos[..., None])
    if c["window"]:
        hidden = hidden | (t <= pos[..., None] - c["window"])
    scores = scores.masked_fill(hidden[None, :, None], float("-inf"))
    top = scores.amax(dim=4, keepdim=True)
    e = torch.exp(scores - top)
    total = e.sum(dim=4, keepdim=True)
    out = torch.matmul(e[..., :c["shared"]].reshape(heads, -1, c["shared"]), v0.permute(1, 0, 2).contiguous()).reshape(heads, seqs, group, new, dim)
    out = out + torch.matmul(e[..., c["shared"]:].reshape(heads, seqs, group * new, -1), v1.permute(2, 0, 1, 3).contiguous()).reshape(out.shape)
    out = (out / total).permute(1, 3, 0, 2, 4).reshape(seqs * new, qh, dim)
    lse = (top + torch.log(total))[..., 0].permute(1, 3, 0, 2).reshape(seqs * new, qh)
    return [out.to(TYPES[c["type"]]), lse.contiguous()]


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


def _round64(x, fmt):
    if fmt == "int8":
        return x.round().clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.clamp((x / step).round() * step, -448, 448)


def _exact_norm(case, s):
    added = s["x"].double() + (s["residual"].double() if case["residual"] else 0)
    gain = s["weight"].double() + case["weight_add"]
    root = torch.sqrt((added * added).sum(dim=1) / case["n"] + EPS)[:, None]
    out = [added * gain / root] if case["y"] else []
    if case["residual"]:
        out.append(added)
    if case["codes"]:
        size = case["group"] or case["n"]
        held = torch.empty_like(added)
        for a in range(0, case["n"], size):
            part = (added * gain)[:, a:a + size]
            unit = part.abs().amax(dim=1, keepdim=True) / (127 if case["codes"] == "int8" else 448)
            if case["codes"] == "fp8":
                unit = torch.exp2(torch.ceil(torch.log2(unit)))
            held[:, a:a + size] = _round64(part / unit, case["codes"]) * unit / root
        out.append(held)
    return out


def _exact_gemm4(case, s):
    n = case["n"]
    x = s["x"].double() if s["x_scales"] is None else _decode64(case["x"], s["x"].view(torch.uint8))
    if s["x_scales"] is not None:
        x = x * s["x_scales"].double()[:, torch.arange(n, device=DEV) // (case["x_group"] or n)]
    y = torch.zeros((case["batch"], case["m"]), dtype=torch.float64, device=DEV)
    for at in range(_groups(n, case["group"])):
        cols = slice(at * case["group"], min(n, (at + 1) * case["group"]))
        y += (x[:, cols] @ s["codes"][:, cols].double().t()) * s["scales"][:, at].double()
    return y


def _exact_logits(case, s):
    vocab = case["vocab"]
    out = torch.empty(s["x"].shape, dtype=torch.float64, device=DEV)
    for q in range(case["seqs"]):
        for i in range(case["rows"]):
            z = s["x"][q, i].double()
            if case["history"]:
                text = s["history"][q, :int(s["lens"][q])].long()
                text, cut = torch.cat([text, s["drafts"][q, :i].long()]), int(s["prompt_lens"][q])
                times = torch.bincount(text[cut:], minlength=vocab)
                before = torch.bincount(text, minlength=vocab) > 0
                by = s["repetition"][q].double()
                z[before] = torch.minimum(z[before] * by, z[before] / by)          # (penalties of at least 1)
                z = z - times * s["frequency"][q].double() - (times > 0) * s["presence"][q].double()
            if case["bias"]:
                z.index_add_(0, s["bias_tokens"][q].long(), s["bias_values"][q].double())
            heat = float(s["temperature"][q])
            z = z / heat if heat > 0 else z
            if case["mask"]:
                word = s["mask"][q, i][torch.arange(vocab, device=DEV) // 32]
                z[(word >> (torch.arange(vocab, device=DEV) % 32)) & 1 == 0] = float("-inf")
            if case["probabilities"]:
                if heat > 0:
                    z = torch.exp(z - torch.logsumexp(z, dim=0))
                else:
                    z = (torch.arange(vocab, device=DEV) == int(torch.nonzero(z == z.max())[0])).double()
            out[q, i] = z
    return out


def _exact_shared(case, s):
    heads, dim, page, new, group = case["heads"], case["dim"], case["page"], case["new"], case["qh"] // case["heads"]
    blocks = page // BLOCK
    size = heads * page * dim
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for seq, own_len in enumerate(s["lengths"]):
        length = case["shared"] + own_len
        pages = s["store"][s["table"][seq, :-(-length // page)].long()]
        n = pages.shape[0]
        scales = pages.view(torch.float32)[:, size // 2:size // 2 + 2 * heads * blocks].double().reshape(n, 2, heads, blocks)
        rows = slice(seq * new, (seq + 1) * new)
        lag = torch.arange(length - new, length, device=DEV)[:, None] - torch.arange(length, device=DEV)
        for h in range(heads):
            part = slice(h * page * dim, (h + 1) * page * dim)
            k = _decode64(case["fmt"], pages[:, part]).reshape(n, blocks, BLOCK, dim) * scales[:, 0, h, :, None, None]
            v = _decode64(case["fmt"], pages[:, size:][:, part]).reshape(n, blocks, dim, BLOCK) * scales[:, 1, h, :, None, None]
            k, v = k.reshape(-1, dim)[:length], v.transpose(2, 3).reshape(-1, dim)[:length]
            mine = slice(h * group, (h + 1) * group)
            z = s["q"][rows, mine].double().reshape(-1, dim) @ k.t().contiguous() / math.sqrt(dim)
            z = z.reshape(new, group, length)
            if case["causal"]:
                z.masked_fill_((lag < 0)[:, None], float("-inf"))
            if case["window"]:
                z.masked_fill_((lag >= case["window"])[:, None], float("-inf"))
            lse[rows, mine] = torch.logsumexp(z, dim=2)
            out[rows, mine] = (torch.exp(z - lse[rows, mine][..., None]).reshape(-1, length) @ v).reshape(new, group, dim)
    return [out, lse]


def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "gemm4": _exact_gemm4, "logits": _exact_logits, "shared": _exact_shared}[case["kind"]](case, s)
