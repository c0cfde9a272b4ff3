"""Sizes at the ends of 32 bits are refused before any launch (CPU: nothing is launched)."""
import pytest
import torch

from test_step_host import A, EINVAL, EUNSUPPORTED, Stream, at, biq, logits  # noqa: F401


def test_histories_whose_places_leave_32_bits(biq):
    """A workgroup counts 2^14 tokens at a time: the next place after the last has to be a number too."""
    lib = biq.load_library()
    for width in ((1 << 31) - 1, (1 << 31) - (1 << 14), (1 << 31) - (1 << 16)):
        assert lib.biq_logits(at(logits(width=width)), A, 1 << 40, None) == EUNSUPPORTED, width
    assert lib.biq_logits(at(logits(width=-1)), A, 1 << 40, None) == EINVAL


def test_tensors_whose_sizes_leave_32_bits(biq):
    """The descriptors' sizes are int: larger ones must not come through as what is left of them.  (Broadcast tensors take no memory.)"""
    many = (1 << 32) + 3
    rows = lambda *shape: torch.zeros(1, *shape[1:]).expand(*shape)
    packed = torch.zeros(biq.biq_packed4_bytes(16, 8, 32), dtype=torch.uint8)
    with pytest.raises(ValueError):
        biq.PreparedNorm(rows(many, 8), rows(many, 8), stream=Stream())
    with pytest.raises(ValueError):
        biq.PreparedGemm4(packed, rows(many, 8), rows(many, 16), 32, stream=Stream())
    with pytest.raises(ValueError):
        biq.biq_gemm4_workspace_bytes(packed, rows(many, 8), rows(many, 16), 32)
    with pytest.raises(ValueError):
        biq.PreparedLogits(rows(many, 1, 8), rows(many, 1, 8), stream=Stream())
    with pytest.raises(ValueError):
        biq.biq_quantize4(rows(many, 8), packed, many, 8, 32, stream=Stream())


def test_logits_whose_rows_would_overlap(biq):
    """Rows of all sequences are written side by side: (strides of a sequence, of a row) that put two of them on the same tokens are refused."""
    lib = biq.load_library()
    status = lambda **change: lib.biq_logits(at(logits(history=None, lens=None, prompt_lens=None, **change)), A, 1 << 40, None)
    how = dict(seqs=4, rows=3, vocab=100, x_seq_stride=300, x_stride=100, mask_seq_stride=12, mask_stride=4)
    for strides in ((100, 100), (299, 100), (100, 399), (250, 500), (150, 100), (200, 300), (1 << 40, 99), (1 << 39, 1 << 40)):
        assert status(out_seq_stride=strides[0], out_stride=strides[1], **how) == EINVAL, strides
    for strides in ((300, 100), (100, 400), (350, 110), (210, 105 * 8), (300, 400), (700, 500), (1 << 40, 100), (100, 1 << 40)):
        assert status(out_seq_stride=strides[0], out_stride=strides[1], **how) not in (EINVAL, EUNSUPPORTED), strides
    one = dict(how, seqs=1)
    assert status(out_seq_stride=0, out_stride=100, **one) not in (EINVAL, EUNSUPPORTED)
    many = dict(how, seqs=40000, rows=50000)
    assert status(out_seq_stride=50000 * 100, out_stride=100, **many) not in (EINVAL, EUNSUPPORTED)
    assert status(out_seq_stride=50000 * 100 - 1, out_stride=100, **many) == EINVAL
    assert status(out_seq_stride=101, out_stride=102, **many) == EINVAL
