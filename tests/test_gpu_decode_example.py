"""examples/speculative_decode.py: the decoder-step operators and the multiply together."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import speculative_decode

    return speculative_decode


@pytest.fixture(scope="module")
def model(ex):
    return ex.Decoder(hidden=256, heads=4, kv_heads=2, dim=64, ffn=512, layers=2, vocab=333, planes=3, positions=512)


PROMPTS = [[1, 2, 3, 4, 5], list(range(70)), [11]]


@pytest.mark.parametrize("format", ["int8", "fp8"])
def test_a_draft_model_that_is_the_target_is_believed(ex, model, format):
    """Same planes: probabilities differ by the order in which the caches were written only."""
    answers, rate, target, draft = ex.generate(model, PROMPTS, 24, drafts=4, draft_planes=3, format=format)
    assert rate > 0.9
    assert all(0 <= t < 333 for a in answers for t in a) and min(len(a) for a in answers) >= 24
    # a cache holds the prompt and all of the answer but its last token
    want = [len(p) + len(a) - 1 for p, a in zip(PROMPTS, answers)]
    assert target[0].lens.tolist() == want and draft[0].lens.tolist() == want


def test_fewer_planes_draft(ex, model):
    answers, rate, _, _ = ex.generate(model, PROMPTS, 16, drafts=3, draft_planes=2)
    assert 0 < rate <= 1 and min(len(a) for a in answers) >= 16
    again, same, _, _ = ex.generate(model, PROMPTS, 16, drafts=3, draft_planes=2)
    assert again == answers and same == rate                    # the same numbers, the same tokens


def test_tokens_one_by_one_see_what_a_prompt_sees(ex, model):
    """The last row's probabilities after a prompt, and after the same tokens fed singly.  The caches' blocks were rounded in another order: a
    code is off by one step (1 / 127 of a block's largest value) at most where a block grew; what that does to probabilities of
    1 / 333 on average is far below them."""
    tokens = torch.tensor(list(range(40)), dtype=torch.int32, device="cuda")
    whole, single = model.caches(1), model.caches(1)
    whole[0].lens.fill_(40)
    p = model.forward(tokens, whole, 3, max_len=40)
    for i in range(40):
        single[0].lens.add_(1)
        q = model.forward(tokens[i:i + 1], single, 3, max_len=40)
    assert (p[-1] - q[0]).abs().max() < 1 / 333
    assert (p[-1] - q[0]).abs().sum() < 0.1
