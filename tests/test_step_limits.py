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
