"""The example's drafted answers: those of one token at a time, whatever the drafts are, in fewer passes where they are good."""

import os
import sys

import numpy as np
import pytest
import torch

import workloads

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import answers as example  # noqa: E402

pytestmark = pytest.mark.gpu


def test_drafted_answers_are_the_plain_ones():
    """fp32, the same random numbers: a token differs only where a sum's rounding (a few thousand times 2^-24) moves a weight across
    the drawn share. Log probabilities are sums of the same terms in another order, below 1e-3 apart."""
    w = example.SMALL
    theta = torch.empty(w.n, dtype=torch.float32, device="cuda")
    workloads.fill_model_buffer_device(theta, w)
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, workloads.QWEN3_VOCAB, n).astype(np.int32) for n in (1, 16, 35)]
    answers, steps = 3, 20
    model = example.Decoder(w, theta, example.pages_needed(prompts, answers, steps))
    u = torch.rand(steps, 9, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    tokens, logprobs = example.answer(model, prompts, answers, u)
    wrong = tokens.clone()
    wrong[:, 5] = (wrong[:, 5] + 1) % workloads.QWEN3_VOCAB  # right up to the fifth token, and from the seventh on
    other = torch.randint(0, workloads.QWEN3_VOCAB, tokens.shape, dtype=torch.int32, device="cuda",
                          generator=torch.Generator(device="cuda").manual_seed(1))
    # the first token comes from the prompt; a pass wins one token and as many drafted ones as agree, up to four
    for drafts, most in (([tokens], 4), ([wrong], 5), ([other], 19), ([], 19), ([other, wrong, tokens], 4), ([tokens[:, :7]], 14)):
        got, lp, passes = example.answer_drafted(model, prompts, answers, u, drafts)
        assert torch.equal(got, tokens) and float((lp - logprobs).abs().max()) < 1e-3
        assert len(passes) == 9 and max(passes) <= most, passes


def test_drafted_example_trains(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["answers.py", "--steps", "1", "--probes", "2", "--answers", "4", "--tokens", "6", "--drafted"])
    example.main()
    assert "passes an answer for 5" in capsys.readouterr().out
