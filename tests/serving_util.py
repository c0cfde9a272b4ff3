"""Plain 64-bit forms of the decoder-step operators and caches to run them on (CPU, numpy and torch)."""
import numpy as np
import torch

BLOCK = 16
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def page_bytes(page, heads, dim):
    return -(-(2 * page * heads * dim + 8 * heads * (page // BLOCK)) // 128) * 128


def fp8_values():
    out = np.zeros(256)
    for b in range(256):
        e, f = (b >> 3) & 15, b & 7
        v = f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        out[b] = (-v if b & 128 else v) if b & 127 != 127 else np.nan
    return out


VALUES = {"int8": np.where(np.arange(256) < 128, np.arange(256), np.arange(256) - 256).astype(float), "fp8": fp8_values()}


def rounded(x, fmt):
    """x (float64) -> nearest number with a code, ties to even."""
    if fmt == "int8":
        return np.clip(np.rint(x), -127, 127)
    a = np.abs(x)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.rint(x / step) * step


def code_of(value, fmt):
    """Bytes of numbers that have a code."""
    if fmt == "int8":
        return value.astype(np.int8).view(np.uint8)
    return torch.from_numpy(value.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def fresh_scale(amax, fmt):
    if amax < 2.0 ** -100:
        return np.float32(0)
    if fmt == "int8":
        return np.float32(amax) * np.float32(1 / 127)
    return np.float32(2.0 ** np.ceil(np.log2(np.float64(amax) / 448.0)))


class Pages:
    """A cache in numpy: bytes as include/biq.h lays them out."""

    def __init__(self, lens, heads, dim, page, fmt, rng, width=None, spare=2):
        self.heads, self.dim, self.page, self.fmt = heads, dim, page, fmt
        need = [-(-n // page) for n in lens]
        width = width or max(need) + 1
        total = sum(need) + spare
        self.store = rng.integers(0, 256, size=(total, page_bytes(page, heads, dim)), dtype=np.uint8)   # garbage, NaN among it
        order = rng.permutation(total).astype(np.int32)
        self.table = np.full((len(lens), width), -7, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.lens = np.array(lens, np.int32)

    def _where(self, s, b, head, which):
        pg, sub = self.table[s, b * BLOCK // self.page], b % (self.page // BLOCK)
        block = (which * self.heads + head) * (self.page // BLOCK) + sub
        at = block * BLOCK * self.dim
        return pg, slice(at, at + BLOCK * self.dim), slice(2 * self.page * self.heads * self.dim + 4 * block, 2 * self.page * self.heads * self.dim + 4 * block + 4)

    def block(self, s, b, head, which):
        """Codes as numbers [16][dim] and the scale."""
        pg, codes, scale = self._where(s, b, head, which)
        v = VALUES[self.fmt][self.store[pg, codes]]
        v = v.reshape(BLOCK, self.dim) if which == 0 else v.reshape(self.dim, BLOCK).T
        return v, self.store[pg, scale].copy().view(np.float32)[0]

    def put(self, s, b, head, which, numbers, scale):
        pg, codes, at = self._where(s, b, head, which)
        self.store[pg, codes] = code_of(numbers if which == 0 else numbers.T, self.fmt).reshape(-1)
        self.store[pg, at] = np.array([scale], np.float32).view(np.uint8)

    def append(self, s, pos0, k, v):
        """Tokens from pos0 on, float64 [n][heads][dim]; rounds as the operator is defined."""
        for which, x in ((0, k), (1, v)):
            n = x.shape[0]
            for b in range(max(pos0, 0) // BLOCK, -(-(pos0 + n) // BLOCK)):
                t = np.arange(b * BLOCK, (b + 1) * BLOCK)
                new = (t >= pos0) & (t < pos0 + n)
                old = t < pos0
                for h in range(self.heads):
                    numbers, scale = np.zeros((BLOCK, self.dim)), np.float32(0)
                    if old.any():
                        numbers, scale = self.block(s, b, h, which)
                    x16 = np.zeros((BLOCK, self.dim), np.float32)
                    x16[new] = x[t[new] - pos0, h]
                    amax = np.abs(x16).max()
                    if not np.isfinite(x16).all() or np.isnan(scale):
                        self.put(s, b, h, which, np.zeros((BLOCK, self.dim)), np.float32("nan"))
                        continue
                    now = max(fresh_scale(amax, self.fmt), scale)
                    y = np.zeros((BLOCK, self.dim), np.float32)
                    if now > 0:
                        y[new] = x16[new] * (np.float32(1) / now)
                        y[old] = numbers[old].astype(np.float32) * (scale / now)
                    self.put(s, b, h, which, rounded(y.astype(np.float64), self.fmt), now)

    def values(self, s, length=None):
        """K, V float64 [len][heads][dim]."""
        n = int(self.lens[s]) if length is None else length
        out = np.zeros((2, -(-max(n, 1) // BLOCK) * BLOCK, self.heads, self.dim))
        for b in range(-(-n // BLOCK)):
            for h in range(self.heads):
                for w in (0, 1):
                    numbers, scale = self.block(s, b, h, w)
                    out[w, b * BLOCK:(b + 1) * BLOCK, h] = numbers * np.float64(scale)
        return out[0, :n], out[1, :n]

    def on(self, biq, device="cuda:0", lens=None):
        to = lambda a: torch.from_numpy(a).to(device)
        return biq.KvCache(to(self.store), to(self.table), to(self.lens if lens is None else np.asarray(lens, np.int32)), self.page,
                           self.heads, self.dim, self.fmt)


def filled(lens, heads, dim, page, fmt, seed, big=1.0):
    """A cache whose tokens are random: a few large channels in the keys, tails in the values."""
    rng = np.random.default_rng(seed)
    c = Pages(lens, heads, dim, page, fmt, rng)
    channel = np.exp(0.7 * rng.standard_normal((heads, dim)))
    for s, n in enumerate(lens):
        if n:
            v = rng.standard_normal((n, heads, dim))
            c.append(s, 0, (rng.standard_normal((n, heads, dim)) * channel * big).astype(np.float32).astype(np.float64),
                     (v * (1 + 0.3 * np.abs(v))).astype(np.float32).astype(np.float64))
    return c


def attention(q, k, v, scale, pos, causal, window):
    """q [rows][qh][dim], k, v [len][heads][dim], pos [rows] -> out, lse, and the largest sum of |scale q k| and |v| (64 bits)."""
    rows, qh, dim = q.shape
    length, heads = k.shape[:2]
    out, lse = np.zeros((rows, qh, dim)), np.full((rows, qh), -np.inf)
    size = 0.0
    t = np.arange(length)
    for h in range(qh):
        kh, vh = k[:, h // (qh // heads)], v[:, h // (qh // heads)]
        for r in range(rows):
            see = np.ones(length, bool)
            if causal:
                see &= t <= pos[r]
            if window:
                see &= t > pos[r] - window
            if not see.any():
                continue
            z = scale * (kh[see] @ q[r, h])
            with np.errstate(invalid="ignore"):
                size = max(size, abs(scale) * np.nanmax(np.abs(kh[see]) @ np.abs(q[r, h])))
                m = z.max()
                e = np.exp(z - m)
                lse[r, h] = m + np.log(e.sum())
                out[r, h] = e @ vh[see] / e.sum()
    return out, lse, size, np.nanmax(np.abs(v)) if length else 0.0


def attention_bounds(typ, out, size, vmax):
    """What rounding may cost, element by element.  Weights off by a relative e each move a mean of values by at most 2 e vmax.
    Scores: 24-bit terms, sums over a head in 32 bits (their error taken as 8 units of the largest sum of magnitudes, eight
    times what a sum of 128 random signs has), one product and the exponential.  bf16: weights rounded to 2^-9; fp16: to 2^-17.
    Then the output's own rounding."""
    e = 2.0 ** -24 * (8 * size + 16)
    weight = {"fp32": 0.0, "fp16": 2.0 ** -17, "bf16": 2.0 ** -9}[typ]
    own = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}[typ]
    return 2 * (e + weight) * vmax + own * np.abs(out) + 2.0 ** -24, e + 2.0 ** -22 * (1 + size)


def turned(x, angles, rot, interleaved, inverse=False):
    """x [rows][heads][dim], angles [rows][rot / 2][2] in float64 as complex numbers."""
    z = angles[..., 0] + 1j * (-angles[..., 1] if inverse else angles[..., 1])
    y = np.array(x, np.float64)
    part = y[..., :rot]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :rot // 2], part[..., rot // 2:])
    w = (a + 1j * b) * z[:, None, :]
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = w.real, w.imag
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = w.real, w.imag
    return y


def verify(p, q, drafts, lens, u):
    """One sequence at a time with Python's integers.  p [s][k + 1][v], q or None: float32 arrays."""
    f = np.float32
    tokens, accepted = np.full((p.shape[0], p.shape[1]), -1, np.int32), np.zeros(p.shape[0], np.int32)
    vocab, k = p.shape[2], p.shape[1] - 1

    def weights(r):
        r = np.where(r > 0, r, f(0))
        return np.minimum(r, f(1)).astype(np.float64) * 2.0 ** 40 // 1

    for s in range(p.shape[0]):
        n = k if lens is None else min(max(int(lens[s]), 0), k)
        j = 0
        while j < n:
            t = int(drafts[s, j])
            if not 0 <= t < vocab:
                break
            qt = f(1) if q is None else q[s, j, t]
            if not u[s, j] * qt < p[s, j, t]:
                break
            j += 1
        rest = p[s, j]
        if j < n:
            if q is None:
                taken = np.zeros(vocab, f)
                if 0 <= drafts[s, j] < vocab:
                    taken[drafts[s, j]] = 1
            else:
                taken = q[s, j]
            with np.errstate(invalid="ignore"):
                rest = p[s, j] - taken
        w = [int(x) for x in weights(rest)]
        if sum(w) == 0:
            w = [int(x) for x in weights(p[s, j])]
        total, x = sum(w), float(u[s, k])
        goal = (min(int(x * 2 ** 31), 2 ** 31 - 1) if x > 0 else 0) * total >> 31
        token, run = -1, 0
        if total:
            for token in range(vocab):
                run += w[token]
                if run > goal:
                    break
        tokens[s, :j] = drafts[s, :j]
        tokens[s, j], accepted[s] = token, j
    return tokens, accepted
