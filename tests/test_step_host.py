"""Host side of the operators at the end of a decoder step: sizes, refusals before any launch, the binding's own checks."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3
A = 0x10000                                                     # an address that is never read, since nothing is launched


@pytest.fixture(scope="module")
def biq():
    import paper_2005_09904_amd as biq
    from paper_2005_09904_amd import build

    if build.is_stale():
        build.build_library()
    biq.load_library()
    return biq


def test_structs_match_the_header():
    """Names and types of the fields in their order."""
    from paper_2005_09904_amd import step

    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "biq.h")).read(), flags=re.S)
    mirrors = {"biq_norm_args": step._NormArgs, "biq_gemm4_args": step._Gemm4Args, "biq_logits_args": step._LogitsArgs}
    kinds = {"int": ctypes.c_int, "float": ctypes.c_float, "int64_t": ctypes.c_int64}
    for name, mirror in mirrors.items():
        body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, text).group(1)
        want = []
        for line in body.split(";"):
            m = re.match(r"\s*(?:const )?(\w+)(\*?)\s+(.*)", line.strip(), flags=re.S)
            if m:
                want += [(field.strip(), ctypes.c_void_p if m.group(2) else kinds[m.group(1)]) for field in m.group(3).split(",")]
        assert list(mirror._fields_) == want, name


def test_packed_bytes(biq):
    assert biq.biq_packed4_bytes(16, 128, 128) == 1024 + 32
    assert biq.biq_packed4_bytes(17, 129, 32) == 4 * (1024 + 128)
    assert biq.biq_packed4_bytes(32000, 4096, 64) == 2000 * 32 * (1024 + 64)
    for bad in ((0, 1, 32), (1, 0, 32), (1, 1, 16), (1, 1, 0), (1, 1, 256), (-1, 1, 32), (1, (1 << 24) + 1, 32), ((1 << 28) + 1, 1, 32)):
        assert biq.biq_packed4_bytes(*bad) == 0


def at(descriptor):
    """Its address, which is good as long as the descriptor is kept."""
    at.kept = descriptor
    return ctypes.addressof(descriptor)


def norm(**change):
    from paper_2005_09904_amd import step

    a = dict(x=A, residual=2 * A, sum=3 * A, weight=A, y=4 * A, codes=A, scales=A, x_stride=64, residual_stride=64, sum_stride=64, y_stride=64, code_stride=64, type=0,
             y_type=0, rows=3, n=64, group=32, format=0, eps=1e-6, weight_add=0.0)
    return step._NormArgs(**{**a, **change})


def test_norm_refuses(biq):
    lib = biq.load_library()
    assert lib.biq_norm(None, None) == EINVAL
    nan, inf = float("nan"), float("inf")
    for bad in (dict(x=None), dict(y=None, codes=None), dict(residual=None), dict(scales=None), dict(type=3), dict(type=-1), dict(y_type=3), dict(rows=0),
                dict(n=0), dict(group=16), dict(group=-32), dict(group=256), dict(format=2), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(weight_add=nan),
                dict(x=A + 2), dict(y=A + 2), dict(y=A + 1, y_type=1), dict(residual=A + 1), dict(sum=A + 3), dict(weight=A + 2), dict(scales=A + 1),
                dict(y=A, y_type=1), dict(y=A, y_stride=65), dict(y=2 * A, y_stride=65), dict(y=2 * A, y_type=2), dict(y=3 * A), dict(sum=A, sum_stride=65),
                dict(sum=2 * A, sum_stride=65),
                dict(x_stride=-1), dict(residual_stride=-1), dict(sum_stride=63), dict(y_stride=0), dict(code_stride=63), dict(x_stride=(1 << 40) + 1)):
        assert lib.biq_norm(at(norm(**bad)), None) == EINVAL, bad
    big = (1 << 24) + 1
    assert lib.biq_norm(at(norm(n=big, sum_stride=big, y_stride=big, code_stride=big)), None) == EUNSUPPORTED


def gemm4(**change):
    from paper_2005_09904_amd import step

    a = dict(weights=A, x=A, x_scales=A, y=A, x_stride=9000, y_stride=100, m=100, n=9000, group=64, batch=40, x_type=3, x_group=64, y_type=0)
    return step._Gemm4Args(**{**a, **change})


def test_products_refuse(biq):
    lib = biq.load_library()

    def status(a, ws=A, size=1 << 40):
        return lib.biq_gemm4(at(a), ws, size, None)

    assert lib.biq_gemm4(None, A, 1 << 40, None) == EINVAL and lib.biq_gemm4_workspace_bytes(None) == 0
    for bad in (dict(weights=None), dict(x=None), dict(y=None), dict(x_scales=None), dict(m=0), dict(n=0), dict(batch=0), dict(group=0), dict(group=48),
                dict(x_type=5), dict(x_type=-1), dict(y_type=3), dict(x_group=16), dict(x_group=-1), dict(weights=A + 8), dict(x_scales=A + 2), dict(y=A + 2),
                dict(x=A + 1, x_type=1), dict(x_stride=-1), dict(y_stride=99)):
        assert status(gemm4(**bad)) == EINVAL, bad
    for bad in (dict(batch=65536), dict(n=(1 << 24) + 1), dict(m=(1 << 28) + 1, y_stride=1 << 29)):
        assert status(gemm4(**bad)) == EUNSUPPORTED, bad
        assert lib.biq_gemm4_workspace_bytes(at(gemm4(**bad))) == 0
    need = lib.biq_gemm4_workspace_bytes(at(gemm4()))
    assert need >= 2 * 40 * 100 * 4
    assert status(gemm4(), A, need - 1) == EWORKSPACE
    assert status(gemm4(), None, need) == EINVAL and status(gemm4(), A + 8, need) == EINVAL
    assert lib.biq_gemm4_workspace_bytes(at(gemm4(batch=1))) == 0


def test_layout_refuses(biq):
    lib = biq.load_library()
    pack = lambda codes=A, scales=A, packed=A, m=3, n=40, group=32: lib.biq_pack4(codes, scales, packed, m, n, group, None)
    quantize = lambda w=A, stride=40, typ=0, packed=A, m=3, n=40, group=32: lib.biq_quantize4(w, stride, typ, packed, m, n, group, None)
    unpack = lambda packed=A, w=A, stride=40, m=3, n=40, group=32: lib.biq_unpack4(packed, w, stride, m, n, group, None)
    for call in (pack, quantize, unpack):
        for bad in (dict(packed=None), dict(packed=A + 8), dict(m=0), dict(n=0), dict(group=16)):
            assert call(**bad) == EINVAL, bad
    for bad in (dict(codes=None), dict(scales=None), dict(scales=A + 2)):
        assert pack(**bad) == EINVAL
    for bad in (dict(w=None), dict(w=A + 2), dict(typ=3), dict(stride=-1)):
        assert quantize(**bad) == EINVAL
    for bad in (dict(w=None), dict(w=A + 2), dict(stride=39)):
        assert unpack(**bad) == EINVAL
    assert pack(n=(1 << 24) + 1) == EUNSUPPORTED


def logits(**change):
    from paper_2005_09904_amd import step

    a = dict(x=A, out=2 * A, x_seq_stride=60000, x_stride=20000, out_seq_stride=60000, out_stride=20000, mask_seq_stride=1877, mask_stride=625, history=A, lens=A,
             prompt_lens=A, drafts=A, repetition=A, presence=A, frequency=A, temperature=A, bias_tokens=A, bias_values=A, mask=A, type=0, out_type=0, seqs=2,
             rows=3, vocab=20000, width=50, biases=4, probabilities=1)
    return step._LogitsArgs(**{**a, **change})


def test_logits_refuse(biq):
    lib = biq.load_library()

    def status(a, ws=A, size=1 << 40):
        return lib.biq_logits(at(a), ws, size, None)

    assert lib.biq_logits(None, A, 1 << 40, None) == EINVAL
    fields = ("history", "lens", "prompt_lens", "drafts", "repetition", "presence", "frequency", "temperature", "bias_tokens", "bias_values", "mask")
    for bad in (dict(x=None), dict(out=None), dict(type=3), dict(out_type=-1), dict(seqs=0), dict(rows=0), dict(vocab=0), dict(x=A + 2), dict(out=A + 1),
                dict(lens=None), dict(history=None), dict(width=0), dict(biases=-1), dict(bias_tokens=None), dict(bias_values=None), dict(out_stride=19999),
                dict(out_seq_stride=0), dict(x_stride=-1), dict(mask_stride=-1), dict(mask_seq_stride=-1), dict(out=A, out_type=1),
                dict(out=A, out_stride=20001), *({f: A + 2} for f in fields)):
        assert status(logits(**bad)) == EINVAL, bad
    for bad in (dict(vocab=(1 << 22) + 1, out_stride=1 << 23, out_seq_stride=1 << 25), dict(biases=4097), dict(seqs=1 << 16, rows=1 << 15)):
        assert status(logits(**bad)) == EUNSUPPORTED, bad
    need = biq.biq_logits_workspace_bytes(2, 3, 20000)
    assert need >= 2 * 3 * 8 and biq.biq_logits_workspace_bytes(2, 3, 4000) == 0
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, (1 << 22) + 1)):
        assert biq.biq_logits_workspace_bytes(*bad) == 0
    assert status(logits(), A, need - 1) == EWORKSPACE
    assert status(logits(), None, need) == EINVAL and status(logits(), A + 8, need) == EINVAL


# ---- the binding's own checks: CPU tensors, prepared and not called ----------------------------------------------

class Stream:
    cuda_stream = 0x7000


def refused(call, good, *changes):
    call(**good)
    for bad in changes:
        with pytest.raises(ValueError):
            call(**{**good, **bad})


def test_norm_tensors(biq):
    t = torch.zeros
    good = dict(x=t(3, 64), y=t(3, 64), weight=t(64), residual=t(3, 64), sum=t(3, 64), codes=t(3, 64, dtype=torch.int8), scales=t(3, 2), group=32, stream=Stream())
    refused(biq.PreparedNorm, good, dict(x=t(3, 64, dtype=torch.float64)), dict(x=t(64)), dict(x=t(3, 128)[:, ::2]), dict(y=t(3, 65)), dict(y=t(64, 3).t()),
            dict(weight=t(63)), dict(weight=t(64, dtype=torch.bfloat16)), dict(residual=t(3, 64, dtype=torch.bfloat16)), dict(residual=t(2, 64)),
            dict(sum=t(3, 64, device="meta")), dict(codes=None), dict(scales=None), dict(codes=t(3, 64, dtype=torch.uint8)), dict(scales=t(3, 3)), dict(x=t(0, 64)))


def test_products_tensors(biq):
    t = torch.zeros
    w = t(biq.biq_packed4_bytes(50, 300, 64), dtype=torch.uint8)
    good = dict(packed=w, x=t(4, 300, dtype=torch.int8), y=t(4, 50), group=64, x_scales=t(4, 3), x_group=128, stream=Stream())
    refused(biq.PreparedGemm4, good, dict(packed=w[:-1]), dict(packed=w.float()), dict(packed=w[::2]), dict(x_scales=None), dict(x=t(4, 300)), dict(x_scales=t(4, 2)),
            dict(y=t(3, 50)), dict(y=t(4, 50, dtype=torch.float64)), dict(group=16), dict(x=t(4, 600, dtype=torch.int8)[:, ::2]),
            dict(workspace=t(8, dtype=torch.uint8, device="meta")))
    with pytest.raises(ValueError):
        biq.biq_pack4(t(50, 299, dtype=torch.int8), t(50, 5), w, 50, 300, 64, stream=Stream())
    with pytest.raises(ValueError):
        biq.biq_quantize4(t(50, 301), w, 50, 300, 64, stream=Stream())
    with pytest.raises(ValueError):
        biq.biq_unpack4(w, t(50, 300, dtype=torch.bfloat16), 50, 300, 64, stream=Stream())


def test_logits_tensors(biq):
    t, i32 = torch.zeros, torch.int32
    good = dict(x=t(2, 3, 100), out=t(2, 3, 100), history=t(2, 9, dtype=i32), lens=t(2, dtype=i32), prompt_lens=t(2, dtype=i32), drafts=t(2, 2, dtype=i32),
                repetition=t(2), presence=t(2), frequency=t(2), temperature=t(2), bias_tokens=t(2, 5, dtype=i32), bias_values=t(2, 5),
                mask=t(2, 3, 4, dtype=i32), stream=Stream())
    refused(biq.PreparedLogits, good, dict(x=t(6, 100)), dict(out=t(2, 3, 101)), dict(out=t(2, 3, 200)[..., ::2]), dict(lens=None), dict(history=None),
            dict(history=t(3, 9, dtype=i32)), dict(lens=t(3, dtype=i32)), dict(drafts=t(2, 3, dtype=i32)), dict(drafts=t(2, 2)), dict(repetition=t(2, 1)),
            dict(temperature=t(2, dtype=torch.float64)), dict(bias_values=None), dict(bias_values=t(2, 4)), dict(mask=t(2, 3, 3, dtype=i32)), dict(mask=t(2, 3, 4)),
            dict(mask=t(2, 3, 8, dtype=i32)[..., ::2]))


# ---- attention with a shared prefix --------------------------------------------------------------------------------

def test_shared_attention_refuses(biq):
    from paper_2005_09904_amd import serving
    from test_serving_host import BAD_CACHES, BAD_RAGGED, BAD_ROWS, attention, cache, ragged, rows

    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "biq.h")).read(), flags=re.S)
    assert re.search(r"typedef struct \{\s*biq_attention_args attention;\s*int shared;\s*\} biq_attention_shared_args;", text)
    assert list(serving._SharedArgs._fields_) == [("attention", serving._AttentionArgs), ("shared", ctypes.c_int)]
    lib = biq.load_library()

    def status(a, shared=64, ws=A, size=1 << 40):
        return lib.biq_attention_shared(at(serving._SharedArgs(a, shared)), ws, size, None)

    assert lib.biq_attention_shared(None, A, 1 << 40, None) == EINVAL and lib.biq_attention_shared_workspace_bytes(None) == 0
    for shared in (0, -32, 16, 33, 160, 1 << 30):               # pages of 32, four of a sequence
        assert status(attention(), shared) == EINVAL
        assert lib.biq_attention_shared_workspace_bytes(at(serving._SharedArgs(attention(), shared))) == 0
    for bad, code in BAD_CACHES:
        assert status(attention(cache=cache(**bad)), 32) == code, bad
    for bad in BAD_RAGGED:
        assert status(attention(ragged=ragged(**bad))) == EINVAL, bad
    for bad in BAD_ROWS:
        assert status(attention(q=rows(**bad))) == EINVAL and status(attention(out=rows(**bad))) == EINVAL, bad
    for bad in (dict(type=3), dict(q_heads=3), dict(q_heads=0), dict(max_len=-1), dict(window=-1), dict(lse=A + 2)):
        assert status(attention(**bad)) == EINVAL, bad
    need = lib.biq_attention_shared_workspace_bytes(at(serving._SharedArgs(attention(), 64)))
    assert need >= 2 * 6 * 4 * 66 * 4                           # two sets of partial results at least
    assert status(attention(), 64, A, need - 1) == EWORKSPACE
    assert status(attention(), 64, None, need) == EINVAL and status(attention(), 64, A + 8, need) == EINVAL
