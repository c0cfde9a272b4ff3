"""biq_logits where whole rows are longer than 16384 tokens (many sequences, no biases), and where a row has more spans than a wave has lanes."""
import numpy as np
import pytest
import torch

import step_util as su
from test_gpu_logits import call, check, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


@pytest.mark.parametrize("typ,out_type", [("fp32", "fp32"), ("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("seqs,rows,vocab", [(128, 1, 16385), (131, 3, 17000), (128, 2, 32768), (128, 2, 32701)])
def test_long_whole_rows(biq, typ, out_type, seqs, rows, vocab):
    """All but biases: history with a prompt, drafts, penalties, temperatures with a greedy sequence among them, masks."""
    x, h = inputs(seqs, rows, vocab, typ, vocab, biases=0)
    h["mask"][3] = 0                                                # a sequence whose mask leaves nothing
    got = call(biq, x, h, out_type, True, pad=vocab % 4)
    assert (got[3] == 0).all()
    keep = [s for s in range(seqs) if s != 3]
    check(x[keep], {k: v[keep] for k, v in h.items()}, got[keep], out_type, True)


def test_long_whole_rows_each_alone_and_in_place(biq):
    seqs, rows, vocab = 128, 2, 20001
    x, h = inputs(seqs, rows, vocab, "fp32", 5, biases=0)
    for part in (("drafts", "frequency"), ("history", "lens", "repetition"), ("mask", "temperature")):
        part = {k: h[k] for k in part}
        check(x, part, call(biq, x, part, "fp32", True), "fp32", True)
    assert torch.equal(call(biq, x, h, "fp32", True), call(biq, x, h, "fp32", True, in_place=True))


def test_long_whole_rows_with_drafts_of_more_than_a_wave(biq):
    x, h = inputs(128, 70, 16400, "bf16", 6, biases=0, mask=False)
    h["drafts"][:] = np.random.default_rng(1).integers(-2, 60, size=h["drafts"].shape)
    got = call(biq, x, h, "fp32", True)
    for s in (0, 1, 64, 127):                                       # (64: greedy)
        check(x[s:s + 1], {k: v[s:s + 1] for k, v in h.items()}, got[s:s + 1], "fp32", True)


@pytest.mark.parametrize("heat", [1.0, 0.0])
def test_long_whole_rows_with_infinities_and_nan(biq, heat):
    seqs, vocab = 128, 30001
    x = torch.randn((seqs, 1, vocab), generator=torch.Generator().manual_seed(3))
    mask = np.full((seqs, 1, -(-vocab // 32)), -1, np.int32)
    x[0, 0, vocab - 1], x[1, 0, 40] = float("nan"), float("nan")
    mask[1, 0, 1] = ~(1 << 8)                                       # (a masked one)
    x[2] = float("-inf")
    x[3, 0, 1000:] = float("-inf")
    p = su.back(call(biq, x, dict(mask=mask, temperature=np.full(seqs, heat, np.float32)), "fp32", True))
    assert np.isnan(p[0]).all() and (p[2] == 0).all()
    x[1, 0, 40] = 0
    rest = [1, 3, 4, 127]
    check(x[rest], dict(mask=mask[rest], temperature=np.full(4, heat, np.float32)), torch.from_numpy(p[rest]), "fp32", True)


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("seqs,rows,vocab", [(1, 1, 131073), (2, 2, 151001), (2, 1, 262147)])
def test_vocabularies_of_more_than_64_spans(biq, typ, seqs, rows, vocab):
    x, h = inputs(seqs, rows, vocab, typ, vocab)
    h["temperature"][:] = 0.8
    check(x, h, call(biq, x, h, "fp32", True), "fp32", True)
    check(x, h, call(biq, x, h, "fp32", False), "fp32", False)
    h["temperature"][:] = 0
    check(x, h, call(biq, x, h, "fp32", True), "fp32", True)


@pytest.mark.parametrize("vocab", [131073, 262147, 1 << 22])
def test_the_last_spans_of_large_vocabularies(biq, vocab):
    """Past the 64th span: the largest, the first of two that are equal, all of the weight, a NaN."""
    x = torch.zeros((5, 1, vocab))
    x[0, 0, vocab - 1] = 30
    x[1, 0, [131072 - 1, vocab - 1]] = 7
    x[2, 0, vocab - 1] = float("nan")
    x[3, 0, :vocab - 1] = float("-inf")
    x[4] = float("-inf")
    for heat in (1.0, 0.0):
        p = su.back(call(biq, x, dict(temperature=np.full(5, heat, np.float32)), "fp32", True))[:, 0]
        assert np.isnan(p[2]).all() and p[3, vocab - 1] == 1 and p[3].sum() == 1 and (p[4] == 0).all()
        if heat == 0:
            assert p[0].argmax() == vocab - 1 and p[0].sum() == 1 and p[1].argmax() == 131071 and p[1].sum() == 1
        else:
            for s, at, z in ((0, [vocab - 1], 30.0), (1, [131071, vocab - 1], 7.0)):
                want = np.full(vocab, np.exp(-z))
                want[at] = 1
                want /= want.sum()
                # (the exponent 6 roundings of z, three exponentials 2 each, a sum of at most 32 terms in a row and 16 levels, 4 more)
                assert (np.abs(p[s] - want) <= 2.0 ** -24 * (6 * z + 58) * want).all()
