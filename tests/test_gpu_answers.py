"""The example that draws answers with every operator of a decode step, against a plain decoder."""

import math
import os
import sys

import numpy as np
import pytest
import torch

import workloads

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import answers as example  # noqa: E402

pytestmark = pytest.mark.gpu


def plain_logits(w, theta, tokens):
    """Logits behind each token of one sequence: the decoder's formulas in float64, no cache."""
    at = {name: theta[o:o + n].double() for name, o, n in workloads.tensor_offsets(w)}
    d, n = workloads.QWEN3_HEAD_DIM, len(tokens)
    norm = lambda x, g: x / torch.sqrt((x * x).mean(-1, keepdim=True) + example.EPS) * g  # noqa: E731
    i = torch.arange(d // 2, dtype=torch.float64, device=theta.device)
    angle = torch.arange(n, device=theta.device)[:, None] * example.ROTARY_BASE ** (-2 * i / d)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    turn = lambda x: torch.cat((x[..., :d // 2] * cos - x[..., d // 2:] * sin, x[..., :d // 2] * sin + x[..., d // 2:] * cos), -1)  # noqa: E731
    embed = at["embed_tokens"].view(-1, w.hidden)
    x = embed[tokens]
    later = torch.ones(n, n, dtype=torch.bool, device=theta.device).triu(1)
    for layer in range(w.layers):
        p = f"layers.{layer}."
        y = norm(x, at[p + "input_norm.gamma"])
        q, k, v = (y @ at[p + f"{c}_proj.weight"].view(-1, w.hidden).T for c in "qkv")
        q = turn(norm(q.view(n, -1, d), at[p + "q_norm.gamma"]))
        k = turn(norm(k.view(n, -1, d), at[p + "k_norm.gamma"])).repeat_interleave(w.heads // w.kv_heads, 1)
        v = v.view(n, -1, d).repeat_interleave(w.heads // w.kv_heads, 1)
        s = (q.transpose(0, 1) @ k.permute(1, 2, 0) / math.sqrt(d)).masked_fill(later, -math.inf)
        o = torch.softmax(s, -1) @ v.transpose(0, 1)
        x = x + o.transpose(0, 1).reshape(n, -1) @ at[p + "o_proj.weight"].view(w.hidden, -1).T
        y = norm(x, at[p + "post_attn_norm.gamma"])
        gate, up = (y @ at[p + f"{c}_proj.weight"].view(-1, w.hidden).T for c in ("gate", "up"))
        x = x + (torch.nn.functional.silu(gate) * up) @ at[p + "down_proj.weight"].view(w.hidden, -1).T
    return norm(x, at["final_norm.gamma"]) @ embed.T


def test_answers_have_the_plain_decoders_probabilities():
    """In fp32 the cached decoder's log probabilities of the tokens it drew (no cuts) are the plain decoder's: two
    layers of sums of 1,024 terms at most are off by a few thousand fp32 roundings, below 1e-3."""
    w = example.SMALL
    theta = torch.empty(w.n, dtype=torch.float32, device="cuda")
    workloads.fill_model_buffer_device(theta, w)
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, workloads.QWEN3_VOCAB, n).astype(np.int32) for n in (1, 16, 35)]
    answers, steps = 3, 20
    model = example.Decoder(w, theta, example.pages_needed(prompts, answers, steps))
    u = torch.rand(steps, 9, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    tokens, logprobs = example.answer(model, prompts, answers, u, top_k=0, top_p=1.0)
    assert tokens.shape == logprobs.shape == (9, steps)
    for a in range(9):
        prompt = torch.from_numpy(prompts[a // answers].astype(np.int64)).cuda()
        logits = plain_logits(w, theta, torch.cat((prompt, tokens[a].long()[:-1])))
        want = torch.log_softmax(logits[len(prompt) - 1:], -1).gather(1, tokens[a].long()[:, None])[:, 0]
        assert float((want - logprobs[a].double()).abs().max()) < 1e-3
    again, _ = example.answer(model, prompts, answers, u, top_k=0, top_p=1.0)
    assert torch.equal(again, tokens)


def test_example_trains_on_its_answers(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["answers.py", "--steps", "1", "--probes", "2", "--answers", "4", "--tokens", "5"])
    example.main()
    assert "step 0: odd tokens" in capsys.readouterr().out
