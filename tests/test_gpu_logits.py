"""biq_logits against 64 bits."""
import numpy as np
import pytest
import torch

import step_util as su

pytestmark = pytest.mark.gpu
INTS = ("history", "lens", "prompt_lens", "drafts", "bias_tokens", "mask")


@pytest.fixture(scope="module")
def biq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2005_09904_amd as biq

    biq.load_library()
    return biq


def inputs(seqs, rows, vocab, typ, seed, history=60, biases=9, mask=True):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((seqs, rows, vocab)).astype(np.float32) * 4).to(su.TYPES[typ])
    token = lambda *shape: rng.integers(0, max(1, min(vocab, 40)), size=shape).astype(np.int32) * max(1, vocab // 40)
    h = {}
    if history:
        h = dict(history=token(seqs, history), lens=rng.integers(0, history + 1, size=seqs).astype(np.int32), drafts=token(seqs, rows - 1))
        h["history"][:, ::7] = rng.integers(-5, vocab + 5, size=h["history"][:, ::7].shape)
        h["prompt_lens"] = (h["lens"] * rng.uniform(0, 1, size=seqs)).astype(np.int32)
        h.update(repetition=rng.uniform(0.7, 1.6, size=seqs), presence=rng.uniform(-0.5, 1, size=seqs), frequency=rng.uniform(-0.3, 0.5, size=seqs))
    h["temperature"] = rng.uniform(0.3, 2, size=seqs)
    h["temperature"][seqs // 2] = 0
    if biases:
        h.update(bias_tokens=token(seqs, biases), bias_values=rng.uniform(-3, 3, size=(seqs, biases)))
        h["bias_tokens"][0, -1] = -1
    if mask:
        h["mask"] = rng.integers(-2 ** 31, 2 ** 31, size=(seqs, rows, -(-vocab // 32))).astype(np.int32)
    return x, {k: v if k in INTS else v.astype(np.float32) for k, v in h.items()}


def call(biq, x, h, out_type, probabilities, pad=0, in_place=False):
    seqs, rows, vocab = x.shape
    tx = torch.full((seqs, rows, vocab + pad), 7.0, dtype=x.dtype, device="cuda:0")[..., :vocab]
    tx.copy_(x)
    out = tx if in_place else torch.full((seqs, rows, vocab + pad), 77.0, dtype=su.TYPES[out_type], device="cuda:0")[..., :vocab]
    ws = torch.full((max(16, biq.biq_logits_workspace_bytes(seqs, rows, vocab)),), 0xff, dtype=torch.uint8, device="cuda:0")
    biq.biq_logits(tx, out, probabilities=probabilities, workspace=ws, **{k: torch.from_numpy(v).to("cuda:0") for k, v in h.items()})
    torch.cuda.synchronize()
    return out


def check(x, h, got, out_type, probabilities):
    """Logits: five roundings (division, product and two subtractions, biases, temperature's reciprocal and product) of numbers up to `size`.
    Probabilities: such differences in the exponent twice, 2^-22 of the exponent for its product with log2 e and the exponential, a sum in 32 bits of
    which at most 16 terms follow one another before trees of 16 levels, a reciprocal and a product."""
    z, greedy = su.logits(x.double().numpy(), **h)
    got = su.back(got)
    size = np.nan_to_num(np.abs(x.double().numpy()), posinf=0) * 1.7 + 3 * 9 + 60 * 0.5 + 1       # (infinities come through unrounded)
    if "temperature" in h:
        t = h["temperature"][:, None, None].astype(np.float64)
        size = size / np.where(t > 0, t, 1)
    off = 2.0 ** -24 * 16 * size
    if not probabilities:
        assert np.array_equal(np.isfinite(got), np.isfinite(z)) and np.array_equal(got[~np.isfinite(z)], z[~np.isfinite(z)])
        fine = np.isfinite(z)
        bound = off + su.HALF[out_type] * np.abs(z) * (1 + 2.0 ** -8)
        assert (np.abs(got[fine] - z[fine]) <= bound[fine]).all()
        return
    p = su.probabilities(z, greedy)
    top = np.where(np.isfinite(z.max(axis=2)), z.max(axis=2), 0)[..., None]
    depth = np.where(np.isfinite(z), top - z, 0)
    rel = 2 * off.max(axis=2, keepdims=True) + 2.0 ** -22 * depth + 2.0 ** -24 * 64
    bound = p * (rel + su.HALF[out_type] * (1 + 2.0 ** -8)) + 2.0 ** -25
    soft = ~greedy
    assert (np.abs(got - p)[soft] <= bound[soft]).all(), np.max(np.abs(got - p)[soft] / bound[soft])
    assert np.array_equal(got[greedy], p[greedy])


@pytest.mark.parametrize("typ,out_type", [("fp32", "fp32"), ("bf16", "fp32"), ("fp16", "fp16"), ("bf16", "bf16")])
@pytest.mark.parametrize("seqs,rows,vocab", [(1, 1, 1), (2, 3, 5), (3, 1, 31), (2, 2, 33), (4, 3, 1000), (3, 4, 4095), (3, 2, 4096), (3, 2, 4097), (5, 3, 9001),
                                             (1, 1, 32000), (1, 2, 70001), (130, 2, 17000)])
@pytest.mark.parametrize("probabilities", [False, True])
def test_all_together(biq, typ, out_type, seqs, rows, vocab, probabilities):
    x, h = inputs(seqs, rows, vocab, typ, seqs + vocab)
    check(x, h, call(biq, x, h, out_type, probabilities, pad=vocab % 4), out_type, probabilities)


@pytest.mark.parametrize("vocab", [700, 9001])
@pytest.mark.parametrize("probabilities", [False, True])
def test_each_alone(biq, vocab, probabilities):
    x, h = inputs(4, 3, vocab, "fp32", vocab)
    tokens = {k: h[k] for k in ("history", "lens")}
    for part in ({}, dict(temperature=h["temperature"]), dict(mask=h["mask"]), dict(bias_tokens=h["bias_tokens"], bias_values=h["bias_values"]),
                 dict(drafts=h["drafts"], frequency=h["frequency"]), dict(repetition=h["repetition"], **tokens), dict(presence=h["presence"], **tokens),
                 dict(frequency=h["frequency"], prompt_lens=h["prompt_lens"], **tokens), tokens):
        check(x, part, call(biq, x, part, "fp32", probabilities), "fp32", probabilities)


@pytest.mark.parametrize("vocab", [900, 9001])
def test_in_place(biq, vocab):
    x, h = inputs(3, 2, vocab, "fp32", 4)
    for probabilities in (False, True):
        assert torch.equal(call(biq, x, h, "fp32", probabilities), call(biq, x, h, "fp32", probabilities, in_place=True))


@pytest.mark.parametrize("vocab", [900, 9001, 40000])
@pytest.mark.parametrize("heat", [1.0, 0.0])
def test_rows_without_tokens_infinities_and_nan(biq, vocab, heat):
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy(rng.standard_normal((6, 1, vocab)).astype(np.float32))
    mask = np.full((6, 1, -(-vocab // 32)), -1, np.int32)
    mask[0] = 0                                                     # nothing is left
    x[1, 0, 5], mask[1, 0, 0] = float("nan"), ~(1 << 5)             # a masked NaN
    x[2, 0, vocab - 1] = float("nan")
    x[3, 0] = float("-inf")
    x[4, 0, 40] = float("-inf")
    x[5, 0, 6], x[5, 0, 7], mask[5, 0, 0] = float("inf"), float("-inf"), ~(1 << 6)      # a masked infinity
    h = dict(mask=mask, temperature=np.full(6, heat, np.float32))
    p = su.back(call(biq, x, h, "fp32", True))
    assert (p[0] == 0).all() and (p[3] == 0).all() and np.isnan(p[2]).all()
    rest = [1, 4, 5]
    sub = {k: v[rest] for k, v in h.items()}
    x = x[rest].clone()
    x[0, 0, 5], x[2, 0, 6] = 0, 0                                   # (hidden: whatever they are)
    check(x, sub, torch.from_numpy(p[rest]), "fp32", True)
    z = su.back(call(biq, x, sub, "fp32", False))
    check(x, sub, torch.from_numpy(z), "fp32", False)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [90, 5001, 16000, 20001])
@pytest.mark.parametrize("heat", [1.0, 0.5, 2.0, 0.0])
def test_the_ends_of_the_type(biq, typ, vocab, heat):
    """Rows all of the type's lowest value, some of it masked, some -infinity; such beside ordinary ones; forced tokens; those banned by a bias."""
    low = torch.finfo(su.TYPES[typ]).min
    x = torch.full((6, 1, vocab), low, dtype=su.TYPES[typ])
    mask = np.full((6, 1, -(-vocab // 32)), -1, np.int32)
    mask[1, 0, 0] = 0x0ffffff0
    x[2, 0, ::3] = float("-inf")
    x[3, 0, vocab - 2] = 1.0
    x[4, 0], x[4, 0, [1, vocab - 1]] = 3.0, -low
    biases = np.full((6, 2), 0.0, np.float32)
    biases[5] = float("-inf")
    h = dict(mask=mask, temperature=np.full(6, heat, np.float32), bias_tokens=np.tile(np.array([0, vocab - 1], np.int32), (6, 1)), bias_values=biases,
             repetition=np.full(6, 1.5, np.float32), history=np.arange(6, dtype=np.int32)[:, None] * 0 + 7, lens=np.ones(6, np.int32))
    h["repetition"][[0, 1]] = 1
    p = su.back(call(biq, x, h, "fp32", True))[:, 0].astype(np.float64)
    want = np.ones((6, vocab))
    want[1, :4] = want[1, 28:32] = 0
    want[2, ::3] = 0
    want[3], want[4] = np.arange(vocab) == vocab - 2, np.isin(np.arange(vocab), [1, vocab - 1])
    want[5, [0, vocab - 1]] = 0
    if heat == 0:
        want = np.arange(vocab) == want.argmax(axis=1)[:, None]
    else:
        want[[2, 5], 7] = 0                                         # (times 1.5 it is far below the others)
    want = want / want.sum(axis=1, keepdims=True)
    # the sum has equal terms (whole numbers, exact), the reciprocal and the product round once each
    assert (np.abs(p - want) <= 2.0 ** -22 * want).all()


def test_the_ends_of_the_type_in_many_whole_rows(biq):
    x = torch.full((128, 1, 20001), torch.finfo(torch.bfloat16).min, dtype=torch.bfloat16)
    x[::2, 0, 5:] = float("-inf")
    p = su.back(call(biq, x, {}, "fp32", True))[:, 0].astype(np.float64)
    assert (np.abs(p[::2] - 0.2 * (np.arange(20001) < 5)) <= 2.0 ** -22).all() and (np.abs(p[1::2] * 20001 - 1) <= 2.0 ** -22).all()


def test_nothing_said_yet_and_no_biases(biq):
    x, h = inputs(2, 2, 700, "fp32", 8)
    none = dict(h, history=np.zeros((2, 0), np.int32), bias_tokens=np.zeros((2, 0), np.int32), bias_values=np.zeros((2, 0), np.float32))
    without = {k: v for k, v in h.items() if k not in ("history", "lens", "prompt_lens", "bias_tokens", "bias_values")}
    assert torch.equal(call(biq, x, none, "fp32", True), call(biq, x, without, "fp32", True))


def test_the_first_of_several_largest(biq):
    for vocab in (50, 5000, 20000):
        x = torch.zeros((3, 1, vocab))
        x[1, 0, [vocab // 2, vocab - 1]] = 2
        x[2, 0, vocab - 1] = 1e-30
        p = call(biq, x, dict(temperature=np.array([0, -1, np.nan], np.float32)), "fp32", True)
        assert p.argmax(dim=2)[:, 0].tolist() == [0, vocab // 2, vocab - 1] and (p.sum(dim=2) == 1).all()


def test_temperatures_at_the_ends(biq):
    """Very hot ones leave all tokens alike, but for masked ones; very cold ones take the likeliest, as do negative ones and NaN."""
    x = torch.randn((6, 1, 20000), generator=torch.Generator().manual_seed(1))
    mask = np.full((6, 1, 625), 0x55555555, np.int32)
    p = su.back(call(biq, x, dict(mask=mask, temperature=np.array([np.inf, 1e38, 1e-35, 1e-28, -1, np.nan], np.float32)), "fp32", True))
    seen = np.arange(20000) % 2 == 0
    for s in range(6):
        assert (p[s, 0, ~seen] == 0).all()
        if s < 2:
            assert np.allclose(p[s, 0, seen], 1e-4, rtol=1e-5)
        else:
            assert p[s, 0].max() == 1 and p[s, 0].sum() == 1 and p[s, 0].argmax() == np.where(seen, x[s, 0].numpy(), -9).argmax()


def test_lengths_and_biases_beyond_their_bounds(biq):
    x, h = inputs(3, 2, 500, "fp32", 5)
    h["lens"] = np.array([-3, 1 << 30, 10], np.int32)
    h["prompt_lens"] = np.array([-1, -(1 << 31), (1 << 31) - 1], np.int32)
    check(x, h, call(biq, x, h, "fp32", False), "fp32", False)


@pytest.mark.parametrize("probabilities", [False, True])
def test_more_rows_than_a_wave_has_lanes(biq, probabilities):
    for vocab in (300, 20000):
        x, h = inputs(2, 140, vocab, "bf16", 6, mask=False)
        h["drafts"][:] = np.random.default_rng(1).integers(-2, 60, size=h["drafts"].shape)
        check(x, h, call(biq, x, h, "fp32", probabilities), "fp32", probabilities)


def test_a_long_history_and_many_biases(biq):
    rng = np.random.default_rng(9)
    x = torch.from_numpy(rng.standard_normal((2, 2, 5000)).astype(np.float32))
    h = dict(history=rng.integers(0, 30, size=(2, 60000)).astype(np.int32), lens=np.array([60000, 33333], np.int32), frequency=np.full(2, 2.0 ** -12, np.float32),
             bias_tokens=rng.integers(0, 5000, size=(2, 4096)).astype(np.int32), bias_values=(rng.integers(-64, 64, size=(2, 4096)) / 64).astype(np.float32))
    z, _ = su.logits(x.double().numpy(), **h)
    got = su.back(call(biq, x, h, "fp32", False))
    assert (np.abs(got - z) <= 2.0 ** -24 * 8 * (np.abs(z) + 40)).all()


def test_drawing_after_them(biq):
    """Probabilities go on to biq_verify_drafts: only tokens that the mask leaves are drawn, none where it leaves nothing."""
    seqs, drafts, vocab = 5, 2, 6000
    x, h = inputs(seqs, drafts + 1, vocab, "bf16", 3)
    h["mask"][2, :] = 0
    p = call(biq, x, h, "fp32", True)
    tokens, accepted = (torch.empty(s, dtype=torch.int32, device="cuda:0") for s in ((seqs, drafts + 1), (seqs,)))
    ws = torch.empty(biq.biq_verify_workspace_bytes(seqs, vocab), dtype=torch.uint8, device="cuda:0")
    biq.biq_verify_drafts(p, None, torch.from_numpy(h["drafts"]).to("cuda:0"), torch.rand((seqs, drafts + 1), device="cuda:0"), tokens, accepted, workspace=ws)
    for s in range(seqs):
        n = int(accepted[s])
        drawn = int(tokens[s, n])
        if s == 2:
            assert n == 0 and drawn == -1
        else:
            assert (int(h["mask"][s, n, drawn // 32]) >> (drawn % 32)) & 1
