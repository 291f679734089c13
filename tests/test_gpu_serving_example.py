"""The serving operators together, as examples/serving_step.py runs them."""

import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 4)])
def test_single_tokens_continue_a_prompt(window, sinks):
    # A text as one prompt, and the same text as a shorter prompt and single
    # tokens.  The two differ by rounding: 8-bit activations of four linears in
    # each of two layers (steps of 2^-7 of a row's largest value, about a
    # hundredth of its size, which add up incoherently), and keys whose page
    # scale grew on the way.  Log probabilities are of size 10 with a spread of
    # about 1: a tenth is five such steps.
    import serving_step as s
    model = s.Model(seed=3, window=window, sinks=sinks)
    g = torch.Generator()
    g.manual_seed(4)
    texts = [torch.randint(0, s.VOCAB, (n,), generator=g, device="cpu").tolist() for n in (140, 75)]
    whole = s.Sequences(2, 150)
    cu, most = whole.extend([140, 75])
    logits = model.step(torch.tensor(texts[0] + texts[1], device="cuda"), cu, most, whole)
    parts = s.Sequences(2, 150)
    cu, most = parts.extend([130, 65])
    got = [model.step(torch.tensor(texts[0][:130] + texts[1][:65], device="cuda"), cu, most, parts)]
    for i in range(10):
        cu, most = parts.extend([1, 1])
        got.append(model.step(torch.tensor([texts[0][130 + i], texts[1][65 + i]], device="cuda"), cu, most, parts))
    for first, n, b in ((0, 140, 0), (140, 75, 1)):
        a = torch.log_softmax(logits[first + n - 10:first + n].float(), 1)
        c = torch.log_softmax(torch.stack([x[b] for x in got[1:]]).float(), 1)
        assert float((a - c).abs().mean()) < 0.1
    assert torch.equal(whole.lengths, parts.lengths)


def test_generate():
    import serving_step as s
    prompts = [[1, 2, 3], list(range(70))]
    answers, steps = s.generate(s.Model(window=64, sinks=2), prompts, 4, top=3)
    again, _ = s.generate(s.Model(window=64, sinks=2), prompts, 4, top=3)
    assert torch.equal(answers, again)                     # nothing depends on an order of arrival
    for i, (logprobs, entropy, top, ids) in enumerate(steps):
        assert torch.equal(ids[:, 0], answers[:, i]) and torch.equal(top[:, 0], logprobs)
        assert bool((logprobs < 0).all()) and bool((entropy > 0).all())
