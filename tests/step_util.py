"""Plain forms of the operators at the end of a decoder step (CPU, numpy), in 64 bits or, where codes have to be equal, rounded
as the operator is defined."""
import numpy as np
import torch

from serving_util import TYPES, rounded  # noqa: F401

HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}          # half a step of 1, relative


def to(a, typ, device="cuda:0"):
    return torch.from_numpy(np.ascontiguousarray(a)).to(TYPES[typ]).to(device)


def back(t):
    return t.detach().cpu().double().numpy()


def groups(n, group):
    return 1 if group == 0 else -(-n // group)


# ---- norm ----------------------------------------------------------------------------------------------------

def norm(x, residual, weight, weight_add, eps):
    """Everything float64: s, r, y."""
    s = x + (0 if residual is None else residual)
    w = (np.ones(x.shape[1]) if weight is None else weight) + weight_add
    with np.errstate(all="ignore"):
        r = 1 / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
        return s, r, s * r * w


def norm_codes(x, residual, weight, weight_add, group, fmt):
    """Codes as numbers and u of every group, each operation rounded to 32 bits.  x, residual, weight float32."""
    f = np.float32
    with np.errstate(all="ignore"):
        s = x if residual is None else x + residual
        w = (np.ones(x.shape[1], f) if weight is None else weight) + f(weight_add)
        t = (s * w).astype(f)
        size = group or x.shape[1]
        codes, units = np.zeros(x.shape), np.zeros((x.shape[0], groups(x.shape[1], group)), f)
        for g in range(units.shape[1]):
            part = t[:, g * size:(g + 1) * size]
            amax = np.abs(part).max(axis=1)
            for i in range(x.shape[0]):
                if not np.isfinite(part[i]).all():
                    units[i, g] = np.nan
                    continue
                if amax[i] < 2.0 ** -100:
                    continue
                u = f(amax[i]) * f(1 / 127) if fmt == "int8" else f(2.0 ** np.ceil(np.log2(np.float64(amax[i]) / 448.0)))
                units[i, g] = u
                codes[i, g * size:(g + 1) * size] = rounded((part[i] * (f(1) / u)).astype(f).astype(np.float64), fmt)
    return codes, units


# ---- products with 4-bit weights -----------------------------------------------------------------------------

def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16().float().numpy()


def spread(scales, n, group):
    return np.repeat(scales, n if group == 0 else group, axis=1)[:, :n]


def quantized4(w, group):
    """Codes and scales of float32 w, rounded as defined."""
    f = np.float32
    m, n = w.shape
    codes, scales = np.zeros((m, n), np.int8), np.zeros((m, groups(n, group)), f)
    for g in range(scales.shape[1]):
        part = w[:, g * group:(g + 1) * group]
        for i in range(m):
            if not np.isfinite(part[i]).all():
                scales[i, g] = np.nan
                continue
            amax = f(np.abs(part[i]).max())
            if amax < 2.0 ** -100:
                continue
            scales[i, g] = bf16(amax * f(1 / 7))
            codes[i, g * group:(g + 1) * group] = np.clip(np.rint(part[i] * (f(1) / scales[i, g])), -8, 7)
    return codes, scales


# ---- logits --------------------------------------------------------------------------------------------------

def logits(x, history=None, lens=None, prompt_lens=None, drafts=None, repetition=None, presence=None, frequency=None, temperature=None,
           bias_tokens=None, bias_values=None, mask=None):
    """x float64 [seqs][rows][vocab] -> adjusted logits in 64 bits, the greedy sequences."""
    z = x.copy()
    seqs, rows, vocab = x.shape
    greedy = np.zeros(seqs, bool)
    with np.errstate(all="ignore"):
        for s in range(seqs):
            for i in range(rows):
                prompt, said = np.zeros(vocab, np.int64), np.zeros(vocab, np.int64)
                if history is not None:
                    n = min(max(int(lens[s]), 0), history.shape[1])
                    for t, token in enumerate(history[s, :n]):
                        if 0 <= token < vocab:
                            (prompt if prompt_lens is not None and t < prompt_lens[s] else said)[token] += 1
                if drafts is not None:
                    for token in drafts[s, :i]:
                        if 0 <= token < vocab:
                            said[token] += 1
                row = z[s, i]
                if repetition is not None:
                    by = float(repetition[s])
                    row = np.where(prompt + said > 0, np.where(row > 0, row / by, row * by), row)
                if frequency is not None:
                    row = np.where(said > 0, row - said * float(frequency[s]), row)
                if presence is not None:
                    row = np.where(said > 0, row - float(presence[s]), row)
                if bias_tokens is not None:
                    for token, value in zip(bias_tokens[s], bias_values[s]):
                        if 0 <= token < vocab:
                            row[token] += float(value)
                if temperature is not None:
                    t = float(temperature[s])
                    greedy[s] = not t > 0
                    row = row if greedy[s] else row / t
                if mask is not None:
                    bits = (mask[s, i].astype(np.int64)[np.arange(vocab) // 32] >> (np.arange(vocab) % 32)) & 1
                    row = np.where(bits > 0, row, -np.inf)
                z[s, i] = row
    return z, greedy


def probabilities(z, greedy):
    p = np.zeros(z.shape)
    with np.errstate(all="ignore"):
        for s in range(z.shape[0]):
            for i in range(z.shape[1]):
                row = z[s, i]
                if np.isnan(row).any():
                    p[s, i] = np.nan
                elif greedy[s]:
                    if row.max() > -np.inf:
                        p[s, i, np.argmax(row)] = 1
                elif row.max() > -np.inf:
                    e = np.exp(row - row.max())
                    p[s, i] = e / e.sum()
    return p
