"""The operators at the end of a decoder step (include/biq.h, its last part): the norm with the residual's addition, products
with 4-bit weights, penalties and masks on logits.  Functions and Prepared* objects as in serving.py: a function looks at its
tensors anew, 10 to 15 us of host time, where calling a prepared object takes 2.5 to 3.5.
"""
from __future__ import annotations

import ctypes

from . import binding
from .serving import FORMATS, I, L, P, _need, _Prepared, _type, _whole

F = ctypes.c_float
INT_MAX = (1 << 31) - 1
X_CODES = {"torch.int8": 3, "torch.float8_e4m3fn": 4}


class _NormArgs(ctypes.Structure):
    _fields_ = [("x", P), ("residual", P), ("sum", P), ("weight", P), ("y", P), ("codes", P), ("scales", P), ("x_stride", L),
                ("residual_stride", L), ("sum_stride", L), ("y_stride", L), ("code_stride", L), ("type", I), ("y_type", I), ("rows", I), ("n", I),
                ("group", I), ("format", I), ("eps", F), ("weight_add", F)]


class _Gemm4Args(ctypes.Structure):
    _fields_ = [("weights", P), ("x", P), ("x_scales", P), ("y", P), ("x_stride", L), ("y_stride", L), ("m", I), ("n", I), ("group", I),
                ("batch", I), ("x_type", I), ("x_group", I), ("y_type", I)]


class _LogitsArgs(ctypes.Structure):
    _fields_ = [("x", P), ("out", P), ("x_seq_stride", L), ("x_stride", L), ("out_seq_stride", L), ("out_stride", L), ("mask_seq_stride", L),
                ("mask_stride", L), ("history", P), ("lens", P), ("prompt_lens", P), ("drafts", P), ("repetition", P), ("presence", P),
                ("frequency", P), ("temperature", P), ("bias_tokens", P), ("bias_values", P), ("mask", P), ("type", I), ("out_type", I), ("seqs", I),
                ("rows", I), ("vocab", I), ("width", I), ("biases", I), ("probabilities", I)]


def _matrix(t, name, shape=None, like=None, device=None):
    """[rows, n] with adjacent elements; its address and stride."""
    _need(t.dim() == 2 and t.numel() > 0, "%s: [rows, elements] expected" % name)
    _need(max(t.shape) <= INT_MAX, "%s: sizes below 2^31 expected" % name)
    _need(t.shape[1] <= 1 or t.stride(1) == 1, "%s: the elements of a row have to be adjacent" % name)
    _need(shape is None or tuple(t.shape) == tuple(shape), "%s: %s expected" % (name, list(shape or ())))
    _need(like is None or t.dtype == like.dtype, "%s: another type" % name)
    _need(device is None or t.device == device, "%s: another device" % name)
    return t.data_ptr(), t.stride(0)


def _groups(n, group):
    return 1 if group == 0 else -(-n // group) if group > 0 else 0


# ---- norm ----------------------------------------------------------------------------------------------------

class PreparedNorm(_Prepared):
    """biq_norm: x [rows, n] -> y [rows, n] of any of the three types and, or codes (int8 or float8_e4m3fn [rows, n]) with scales
    float32 [rows, groups]; residual and sum like x; weight float32 [n]; group: elements that share a scale (0: the row)."""

    def __init__(self, x, y=None, weight=None, residual=None, sum=None, codes=None, scales=None, group=0, eps=1e-6, weight_add=0.0, stream=None):
        a = _NormArgs(type=_type(x), rows=x.shape[0], n=x.shape[-1], group=group, eps=eps, weight_add=weight_add)
        a.x, a.x_stride = _matrix(x, "x")
        if residual is not None:
            a.residual, a.residual_stride = _matrix(residual, "residual", x.shape, x, x.device)
        if sum is not None:
            a.sum, a.sum_stride = _matrix(sum, "sum", x.shape, x, x.device)
        if weight is not None:
            a.weight = _whole(weight, "weight", "float32", [x.shape[1]], x.device)
        if y is not None:
            a.y, a.y_stride = _matrix(y, "y", x.shape, None, x.device)
            a.y_type = _type(y)
        _need((codes is None) == (scales is None), "codes and scales come together")
        if codes is not None:
            _need(str(codes.dtype) in X_CODES, "codes: int8 or float8_e4m3fn expected")
            a.codes, a.code_stride = _matrix(codes, "codes", x.shape, None, x.device)
            a.format = FORMATS["int8" if str(codes.dtype) == "torch.int8" else "fp8"]
            a.scales = _whole(scales, "scales", "float32", [x.shape[0], _groups(x.shape[1], group)], x.device)
        super().__init__("biq_norm", a, (x, y, weight, residual, sum, codes, scales), stream=stream)


def biq_norm(x, y=None, weight=None, residual=None, sum=None, codes=None, scales=None, group=0, eps=1e-6, weight_add=0.0, stream=None) -> None:
    PreparedNorm(x, y, weight, residual, sum, codes, scales, group, eps, weight_add, stream)()


# ---- products with 4-bit weights -----------------------------------------------------------------------------

def biq_packed4_bytes(m: int, n: int, group: int) -> int:
    return binding.load_library().biq_packed4_bytes(m, n, group)


def _packed(packed, m, n, group, device):
    _need(str(packed.dtype) == "torch.uint8" and packed.is_contiguous() and packed.device == device, "packed: dense uint8 on %s expected" % device)
    need = biq_packed4_bytes(m, n, group)
    _need(need > 0, "group: 32, 64 or 128")
    _need(packed.numel() >= need, "packed: %d bytes expected" % need)
    return packed.data_ptr()


def biq_pack4(codes, scales, packed, m: int, n: int, group: int, stream=None) -> None:
    """codes int8 [m, n] in -8 .. 7, scales float32 [m, groups] -> packed."""
    to = _packed(packed, m, n, group, codes.device)
    binding._check(binding.load_library().biq_pack4(_whole(codes, "codes", "int8", [m, n], codes.device),
                                                    _whole(scales, "scales", "float32", [m, _groups(n, group)], codes.device), to, m, n, group,
                                                    binding._stream(stream)), "biq_pack4")


def biq_quantize4(W, packed, m: int, n: int, group: int, stream=None) -> None:
    """W [m, n] -> packed, by the largest magnitude of each group."""
    at, stride = _matrix(W, "W", [m, n])
    binding._check(binding.load_library().biq_quantize4(at, stride, _type(W), _packed(packed, m, n, group, W.device), m, n, group,
                                                        binding._stream(stream)), "biq_quantize4")


def biq_unpack4(packed, W, m: int, n: int, group: int, stream=None) -> None:
    """The values of packed weights, W float32 [m, n]."""
    at, stride = _matrix(W, "W", [m, n])
    _need(_type(W) == 0, "W: float32 expected")
    binding._check(binding.load_library().biq_unpack4(_packed(packed, m, n, group, W.device), at, stride, m, n, group, binding._stream(stream)),
                   "biq_unpack4")


def _gemm4_args(packed, x, y, group, x_scales, x_group):
    code = X_CODES.get(str(x.dtype))
    a = _Gemm4Args(m=y.shape[-1], n=x.shape[-1], group=group, batch=x.shape[0], x_type=_type(x) if code is None else code, x_group=x_group,
                   y_type=_type(y))
    a.x, a.x_stride = _matrix(x, "x")
    a.y, a.y_stride = _matrix(y, "y", [x.shape[0], y.shape[-1]], None, x.device)
    a.weights = _packed(packed, a.m, a.n, group, x.device)
    _need((x_scales is None) == (code is None), "x_scales belong to codes")
    if x_scales is not None:
        a.x_scales = _whole(x_scales, "x_scales", "float32", [x.shape[0], _groups(x.shape[1], x_group)], x.device)
    return a


def biq_gemm4_workspace_bytes(packed, x, y, group, x_scales=None, x_group=0) -> int:
    """Bytes for PreparedGemm4 / biq_gemm4 with the same arguments."""
    a = _gemm4_args(packed, x, y, group, x_scales, x_group)
    return binding.load_library().biq_gemm4_workspace_bytes(ctypes.addressof(a))


class PreparedGemm4(_Prepared):
    """biq_gemm4: y [batch, m] = x [batch, n] times the packed weights [m, n]; x float32, bfloat16, float16, or codes (int8, float8_e4m3fn) with
    x_scales float32 [batch, groups] and x_group as biq_norm writes them."""

    def __init__(self, packed, x, y, group, x_scales=None, x_group=0, workspace=None, stream=None):
        a = _gemm4_args(packed, x, y, group, x_scales, x_group)
        super().__init__("biq_gemm4", a, (packed, x, y, x_scales), workspace, True, x.device, stream)


def biq_gemm4(packed, x, y, group, x_scales=None, x_group=0, workspace=None, stream=None) -> None:
    PreparedGemm4(packed, x, y, group, x_scales, x_group, workspace, stream)()


# ---- logits --------------------------------------------------------------------------------------------------

def biq_logits_workspace_bytes(seqs: int, rows: int, vocab: int) -> int:
    return binding.load_library().biq_logits_workspace_bytes(seqs, rows, vocab)


class PreparedLogits(_Prepared):
    """biq_logits: x [seqs, rows, vocab] -> out (any of the three types; may be x).  history int32 [seqs, width] with lens and prompt_lens int32
    [seqs], drafts int32 [seqs, rows - 1]; repetition, presence, frequency, temperature float32 [seqs]; bias_tokens int32 and
    bias_values float32 [seqs, biases]; mask int32 [seqs, rows, ceil(vocab / 32)], of any strides between rows."""

    def __init__(self, x, out, history=None, lens=None, prompt_lens=None, drafts=None, repetition=None, presence=None, frequency=None, temperature=None,
                 bias_tokens=None, bias_values=None, mask=None, probabilities=False, workspace=None, stream=None):
        for t, name in ((x, "x"), (out, "out")):
            _need(t.dim() == 3 and t.numel() > 0 and (t.shape[2] <= 1 or t.stride(2) == 1), "%s: [seqs, rows, vocab] with adjacent tokens expected" % name)
            _need(max(t.shape) <= INT_MAX, "%s: sizes below 2^31 expected" % name)
        _need(out.shape == x.shape and out.device == x.device, "out: %s on %s expected" % (list(x.shape), x.device))
        seqs, rows, vocab = x.shape
        a = _LogitsArgs(x=x.data_ptr(), out=out.data_ptr(), x_seq_stride=x.stride(0), x_stride=x.stride(1), out_seq_stride=out.stride(0),
                        out_stride=out.stride(1), type=_type(x), out_type=_type(out), seqs=seqs, rows=rows, vocab=vocab,
                        probabilities=int(bool(probabilities)))
        _need((history is None) == (lens is None), "history and lens come together")
        if history is not None:
            _need(history.dim() == 2 and history.shape[1] <= INT_MAX, "history: [seqs, tokens] expected, fewer than 2^31")
            a.width = history.shape[1]
            a.history = _whole(history, "history", "int32", [seqs, a.width], x.device)
            if a.width == 0:                                        # nothing said yet
                history = lens = prompt_lens = None
        for name, t, kind, shape in (("lens", lens, "int32", [seqs]), ("prompt_lens", prompt_lens, "int32", [seqs]),
                                     ("drafts", drafts, "int32", [seqs, rows - 1]), ("repetition", repetition, "float32", [seqs]),
                                     ("presence", presence, "float32", [seqs]), ("frequency", frequency, "float32", [seqs]),
                                     ("temperature", temperature, "float32", [seqs])):
            if t is not None:
                setattr(a, name, _whole(t, name, kind, shape, x.device) or None)
        _need((bias_tokens is None) == (bias_values is None), "bias_tokens and bias_values come together")
        if bias_tokens is not None:
            _need(bias_tokens.dim() == 2 and bias_tokens.shape[1] <= INT_MAX, "bias_tokens: [seqs, biases] expected, fewer than 2^31")
            a.biases = bias_tokens.shape[1]
            a.bias_tokens = _whole(bias_tokens, "bias_tokens", "int32", [seqs, a.biases], x.device)
            a.bias_values = _whole(bias_values, "bias_values", "float32", [seqs, a.biases], x.device)
        if mask is not None:
            words = -(-vocab // 32)
            _need(str(mask.dtype) == "torch.int32" and tuple(mask.shape) == (seqs, rows, words) and (words == 1 or mask.stride(2) == 1) and
                  mask.device == x.device, "mask: int32 %s on %s expected" % ([seqs, rows, words], x.device))
            a.mask, a.mask_seq_stride, a.mask_stride = mask.data_ptr(), mask.stride(0), mask.stride(1)
        super().__init__("biq_logits", a, (x, out, history, lens, prompt_lens, drafts, repetition, presence, frequency, temperature, bias_tokens,
                                           bias_values, mask), workspace, True, x.device, stream)


def biq_logits(x, out, history=None, lens=None, prompt_lens=None, drafts=None, repetition=None, presence=None, frequency=None, temperature=None,
               bias_tokens=None, bias_values=None, mask=None, probabilities=False, workspace=None, stream=None) -> None:
    PreparedLogits(x, out, history, lens, prompt_lens, drafts, repetition, presence, frequency, temperature, bias_tokens, bias_values, mask,
                   probabilities, workspace, stream)()
