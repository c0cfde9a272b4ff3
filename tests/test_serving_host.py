"""Host side of the decoder-step operators: sizes, frequencies, refusals before any launch, the binding's own checks."""
import ctypes
import math
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3


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
    from paper_2005_09904_amd import serving

    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "biq.h")).read(), flags=re.S)
    mirrors = {"biq_rows": serving._Rows, "biq_rotation": serving._Rotation, "biq_cache": serving._Cache, "biq_ragged": serving._Ragged,
               "biq_rotary_args": serving._RotaryArgs, "biq_cache_append_args": serving._AppendArgs, "biq_cache_read_args": serving._ReadArgs,
               "biq_attention_args": serving._AttentionArgs, "biq_verify_args": serving._VerifyArgs}
    kinds = {"int": ctypes.c_int, "float": ctypes.c_float, "int64_t": ctypes.c_int64}
    for name, mirror in mirrors.items():
        body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, text).group(1)
        want = []
        for line in body.split(";"):
            m = re.match(r"\s*(?:const )?(\w+)(\*?)\s+(.*)", line.strip(), flags=re.S)
            if not m:
                continue
            for field in m.group(3).split(","):
                want.append((field.strip(), ctypes.c_void_p if m.group(2) else mirrors.get(m.group(1)) or kinds[m.group(1)]))
        assert list(mirror._fields_) == want, name


def test_page_bytes(biq):
    assert biq.biq_cache_page_bytes(64, 8, 128) == 2 * 64 * 8 * 128 + 2 * 4 * 8 * 4
    assert biq.biq_cache_page_bytes(16, 1, 16) == 640           # 2 * 256 + 8, to the next 128
    for bad in ((0, 1, 64), (8, 1, 64), (272, 1, 64), (16, 0, 64), (16, 1, 8), (16, 1, 272), (24, 1, 64), (16, 1, 72), (16, -1, 64)):
        assert biq.biq_cache_page_bytes(*bad) == 0


def test_frequencies(biq):
    plain = biq.biq_rotary_frequencies(64, 10000.0)
    for i in (0, 1, 17, 31):
        assert plain[i].item() == pytest.approx(10000.0 ** (-2 * i / 64) / (2 * math.pi), rel=1e-14)
    assert torch.equal(biq.biq_rotary_frequencies(64, 10000.0, "linear", 4.0), plain / 4)
    wide = biq.biq_rotary_frequencies(64, 10000.0, "base", 4.0)
    assert wide[0] == plain[0] and wide[-1].item() == pytest.approx(plain[-1].item() / 4, rel=1e-13)
    parts = biq.biq_rotary_frequencies(64, 10000.0, "by_parts", 4.0, trained=2048, slow=1.0, fast=32.0)
    for i in range(32):
        turns = plain[i].item() * 2048
        keep = min(max((turns - 1) / 31, 0), 1)
        assert parts[i].item() == pytest.approx(plain[i].item() * (keep + (1 - keep) / 4), rel=1e-13)
    assert parts[0] == plain[0] and parts[-1].item() == plain[-1].item() / 4
    nan, inf = float("nan"), float("inf")
    for bad in (dict(rot=0), dict(rot=7), dict(rot=-2), dict(base=1.0), dict(base=nan), dict(base=inf), dict(scaling="linear", factor=0.5),
                dict(scaling="linear", factor=nan), dict(scaling="base", factor=2.0, rot=2), dict(scaling="by_parts", trained=0),
                dict(scaling="by_parts", slow=3.0, fast=3.0), dict(scaling="by_parts", slow=nan)):
        with pytest.raises(biq.BiqError) as e:
            biq.biq_rotary_frequencies(**{"rot": 64, **bad})
        assert e.value.status == EINVAL
    with pytest.raises(ValueError):
        biq.biq_rotary_frequencies(64, scaling="other")


# ---- refusals: addresses that are never read, since nothing is launched ---------------------------------------

A = 0x10000


def rows(row=512, head=64, data=A):
    from paper_2005_09904_amd import serving

    return serving._Rows(data, row, head)


def cache(**change):
    from paper_2005_09904_amd import serving

    c = dict(store=A, table=A, lens=A, num_pages=10, page_tokens=32, table_stride=4, seqs=2, heads=2, head_dim=64, format=0)
    return serving._Cache(**{**c, **change})


def ragged(starts=A, rows=6, max_rows=3):
    from paper_2005_09904_amd import serving

    return serving._Ragged(starts, rows, max_rows)


def attention(**change):
    from paper_2005_09904_amd import serving

    a = dict(cache=cache(), q=rows(), out=rows(), lse=None, ragged=ragged(), type=0, q_heads=4, max_len=128, causal=1, window=0, scale=1.0)
    return serving._AttentionArgs(**{**a, **change})


BAD_CACHES = [(dict(store=None), EINVAL), (dict(table=None), EINVAL), (dict(lens=None), EINVAL), (dict(store=A + 8), EINVAL),
              (dict(table=A + 2), EINVAL), (dict(num_pages=0), EINVAL), (dict(page_tokens=0), EINVAL), (dict(page_tokens=8), EUNSUPPORTED),
              (dict(page_tokens=272), EUNSUPPORTED), (dict(head_dim=40), EUNSUPPORTED), (dict(head_dim=272), EUNSUPPORTED),
              (dict(head_dim=0), EINVAL), (dict(heads=0), EINVAL), (dict(seqs=0), EINVAL), (dict(table_stride=0), EINVAL),
              (dict(format=2), EINVAL), (dict(format=-1), EINVAL), (dict(table_stride=1 << 27), EUNSUPPORTED)]
BAD_RAGGED = [dict(rows=0), dict(max_rows=0), dict(max_rows=7), dict(starts=A + 1), dict(starts=None, max_rows=2), dict(rows=-3)]
BAD_ROWS = [dict(data=None), dict(data=A + 2), dict(row=-1), dict(head=-64), dict(row=(1 << 31) + 1)]


def test_attention_refuses(biq):
    lib = biq.load_library()

    def status(a, ws=A, size=1 << 40):
        return lib.biq_attention(None if a is None else ctypes.addressof(a), ws, size, None)

    assert status(None) == EINVAL and lib.biq_attention_workspace_bytes(None) == 0
    for change, want in BAD_CACHES:
        a = attention(cache=cache(**change))
        assert status(a) == want, change
        assert lib.biq_attention_workspace_bytes(ctypes.addressof(a)) == 0
    for change in BAD_RAGGED:
        assert status(attention(ragged=ragged(**change))) == EINVAL, change
    for change in BAD_ROWS:
        assert status(attention(q=rows(**change))) == EINVAL and status(attention(out=rows(**change))) == EINVAL, change
    for change in (dict(type=3), dict(type=-1), dict(q_heads=0), dict(q_heads=3), dict(max_len=-1), dict(window=-1), dict(lse=A + 2)):
        assert status(attention(**change)) == EINVAL, change
    long = attention(cache=cache(table_stride=4096), ragged=ragged(None, 2, 1), max_len=131072)
    need = lib.biq_attention_workspace_bytes(ctypes.addressof(long))
    assert need > 0
    assert status(long, A, need - 1) == EWORKSPACE and status(long, None, need) == EINVAL and status(long, A + 8, need) == EINVAL


def test_cache_calls_refuse(biq):
    from paper_2005_09904_amd import serving

    lib = biq.load_library()

    def append(**change):
        a = dict(cache=cache(), k=rows(), v=rows(), ragged=ragged(), rotation=serving._Rotation(None, 0, 0, 0), type=0)
        a = serving._AppendArgs(**{**a, **change})
        return lib.biq_cache_append(ctypes.addressof(a), None)

    def read(**change):
        a = dict(cache=cache(), k=rows(), v=rows(), ragged=ragged(), type=0)
        a = serving._ReadArgs(**{**a, **change})
        return lib.biq_cache_read(ctypes.addressof(a), None)

    assert lib.biq_cache_append(None, None) == EINVAL and lib.biq_cache_read(None, None) == EINVAL
    for call in (append, read):
        for change, want in BAD_CACHES:
            assert call(cache=cache(**change)) == want, change
        for change in BAD_RAGGED:
            assert call(ragged=ragged(**change)) == EINVAL, change
        for change in BAD_ROWS:
            assert call(k=rows(**change)) == EINVAL and call(v=rows(**change)) == EINVAL, change
        assert call(type=3) == EINVAL
    for bad in ((A + 4, 9, 64, 0), (A, 0, 64, 0), (A, 9, 63, 0), (A, 9, 66, 0), (A, 9, 0, 0)):
        assert append(rotation=serving._Rotation(*bad)) == EINVAL, bad


def test_rotary_refuses(biq):
    from paper_2005_09904_amd import serving

    lib = biq.load_library()

    def call(**change):
        a = dict(x=rows(), y=rows(data=A + 4096), positions=A, rotation=serving._Rotation(A, 9, 64, 0), type=0, rows=2, heads=2, head_dim=64,
                 inverse=0)
        a = serving._RotaryArgs(**{**a, **change})
        return lib.biq_rotary(ctypes.addressof(a), None)

    assert lib.biq_rotary(None, None) == EINVAL
    for change in BAD_ROWS:
        assert call(x=rows(**change)) == EINVAL and call(y=rows(**change)) == EINVAL, change
    for change in (dict(type=5), dict(rows=0), dict(heads=0), dict(head_dim=0), dict(positions=None), dict(positions=A + 2), dict(head_dim=62),
                   dict(y=rows(row=1024)), dict(x=rows(), y=rows(head=128))):
        assert call(**change) == EINVAL, change
    for bad in ((None, 9, 64, 0), (A + 4, 9, 64, 0), (A, 0, 64, 0), (A, 9, 63, 0), (A, 9, 0, 0)):
        assert call(rotation=serving._Rotation(*bad)) == EINVAL, bad
    assert call(rows=(1 << 31) - 1, heads=1 << 20, y=rows(data=A + 4096)) == EUNSUPPORTED
    for bad in ((None, A, 64, 0, 5, 1.0), (A, None, 64, 0, 5, 1.0), (A + 4, A, 64, 0, 5, 1.0), (A, A + 2, 64, 0, 5, 1.0), (A, A, 63, 0, 5, 1.0),
                (A, A, 0, 0, 5, 1.0), (A, A, 64, -1, 5, 1.0), (A, A, 64, 0, 0, 1.0), (A, A, 64, 0, 5, float("nan"))):
        assert lib.biq_rotary_table(*bad, None) == EINVAL, bad
    assert lib.biq_rotary_table(A, A, 64, (1 << 31) - 5, 100, 1.0, None) == EUNSUPPORTED


def test_verify_refuses(biq):
    from paper_2005_09904_amd import serving

    lib = biq.load_library()

    def call(ws=A, size=1 << 40, **change):
        a = dict(p=A, q=A, p_seq_stride=4000, p_stride=1000, q_seq_stride=3000, q_stride=1000, draft_tokens=A, draft_lens=None, uniform=A,
                 tokens=A, accepted=A, type=0, seqs=2, drafts=3, vocab=1000)
        a = serving._VerifyArgs(**{**a, **change})
        return lib.biq_verify_drafts(ctypes.addressof(a), ws, size, None)

    assert lib.biq_verify_drafts(None, A, 1 << 40, None) == EINVAL
    for change in (dict(p=None), dict(p=A + 2), dict(q=A + 1), dict(draft_tokens=None), dict(draft_tokens=A + 2), dict(draft_lens=A + 1),
                   dict(uniform=None), dict(uniform=A + 2), dict(tokens=None), dict(accepted=None), dict(type=3), dict(seqs=0),
                   dict(drafts=-1), dict(vocab=0), dict(p_stride=-1), dict(q_seq_stride=-1), dict(ws=A + 8, vocab=1 << 20)):
        assert call(**change) == EINVAL, change
    for change in (dict(drafts=64), dict(vocab=(1 << 22) + 1), dict(seqs=(1 << 20) + 1)):
        assert call(**change) == EUNSUPPORTED, change
    need = biq.biq_verify_workspace_bytes(2, 1 << 20)
    assert need > 0 and call(size=need - 1, vocab=1 << 20) == EWORKSPACE
    assert biq.biq_verify_workspace_bytes(0, 5) == 0 and biq.biq_verify_workspace_bytes(5, 0) == 0
    assert biq.biq_verify_workspace_bytes(1, (1 << 22) + 1) == 0


def test_the_binding_refuses_what_does_not_fit_together(biq):
    """Tensors on the host: every check comes before a call."""
    page = biq.biq_cache_page_bytes(32, 2, 64)
    store, table, lens = torch.zeros((5, page), dtype=torch.uint8), torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    c = biq.KvCache(store, table, lens, 32, 2, 64)
    for bad in ((store[:, :-1], table, lens), (store, table.long(), lens), (store, table, lens.float()), (store, table[0], lens),
                (store, table, torch.zeros(3, dtype=torch.int32)), (store.float(), table, lens), (store, table[:, ::2], lens)):
        with pytest.raises(ValueError):
            biq.KvCache(*bad, 32, 2, 64)
    with pytest.raises(ValueError):
        biq.KvCache(store, table, lens, 32, 2, 64, "int4")
    with pytest.raises(ValueError):
        biq.KvCache(store, table, lens, 20, 2, 64)
    q = torch.zeros((2, 4, 64))
    angles = torch.zeros((9, 32, 2))
    for call in (lambda: biq.PreparedAttention(c, q[..., ::2], q), lambda: biq.PreparedAttention(c, q, q[:1]),
                 lambda: biq.PreparedAttention(c, q, q.bfloat16()), lambda: biq.PreparedAttention(c, q.double(), q.double()),
                 lambda: biq.PreparedAttention(c, q.transpose(1, 2), q), lambda: biq.PreparedAttention(c, torch.zeros((3, 4, 64)), torch.zeros((3, 4, 64))),
                 lambda: biq.PreparedAttention(c, q, q, lse=torch.zeros((2, 3))), lambda: biq.PreparedAttention(c, q, q, max_rows=2),
                 lambda: biq.PreparedAttention(c, q, q, starts=torch.zeros(2, dtype=torch.int32)),
                 lambda: biq.PreparedAppend(c, q, q), lambda: biq.PreparedAppend(c, q[:, :2], q[:, :2].half()),
                 lambda: biq.PreparedAppend(c, q[:, :2], q[:, :2], angles=angles.double()), lambda: biq.PreparedRead(c, q[:, :2], q[:1, :2]),
                 lambda: biq.PreparedRotary(q, q, torch.zeros(2), angles), lambda: biq.PreparedRotary(q, q, torch.zeros(3, dtype=torch.int32), angles),
                 lambda: biq.PreparedRotary(q, q, torch.zeros(2, dtype=torch.int32), angles[..., 0]),
                 lambda: biq.PreparedVerify(q, q, torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 4)), torch.zeros((2, 4), dtype=torch.int32),
                                            torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()


def test_statuses_come_back_through_the_prepared_call(biq):
    class Stream:
        cuda_stream = 0x7000

    x, y = torch.zeros((2, 2, 64)), torch.zeros((2, 4, 64))[:, ::2]
    call = biq.PreparedRotary(x, y, torch.zeros(2, dtype=torch.int32), torch.zeros((9, 33, 2)), stream=Stream())   # more pairs than the head has
    for _ in range(2):
        with pytest.raises(biq.BiqError, match="biq_rotary") as e:
            call()
        assert e.value.status == EINVAL
    with pytest.raises(TypeError):
        call._call(1)


def test_token_numbers_beyond_32_bits_are_refused(biq):
    from paper_2005_09904_amd import serving

    lib = biq.load_library()
    big = cache(table_stride=(1 << 26) - 1000)                  # 2^31 tokens but 32000
    a = attention(cache=big, ragged=ragged(A, 40000, 40000))
    assert lib.biq_attention(ctypes.addressof(a), A, 1 << 40, None) == EUNSUPPORTED
    b = serving._AppendArgs(cache=big, k=rows(), v=rows(), ragged=ragged(A, 40000, 40000), rotation=serving._Rotation(None, 0, 0, 0), type=0)
    assert lib.biq_cache_append(ctypes.addressof(b), None) == EUNSUPPORTED
    c = serving._ReadArgs(cache=big, k=rows(), v=rows(), ragged=ragged(A, 40000, 40000), type=0)
    assert lib.biq_cache_read(ctypes.addressof(c), None) == EUNSUPPORTED
