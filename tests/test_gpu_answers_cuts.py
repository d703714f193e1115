"""The example as it ships: bf16 weights, draws cut by top-k and top-p.

Tolerance of the logits. On the way to them about 30 tensors are rounded to bf16, 13 in each of two layers, each by at most 2^-9 of its
values. A gated product and the attention's weights double what reaches them; were all of it to add up, it would be 64 2^-9 = 1/8 of
the logits' spread."""

import os
import sys

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
import workloads
from oracle import decode as oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path[:0] = [os.path.join(ROOT, "examples"), os.path.join(ROOT, "tests")]
import answers as example  # noqa: E402
from test_gpu_answers import plain_logits  # noqa: E402

pytestmark = pytest.mark.gpu


def test_bf16_answers_with_cuts(monkeypatch):
    """Every draw's logits are the plain decoder's behind the prompt and the tokens drawn before, and its token and log probability the
    oracle's for those logits."""
    w = example.SMALL
    theta = torch.empty(w.n, dtype=torch.bfloat16, device="cuda")
    workloads.fill_model_buffer_device(theta, w)
    rng = np.random.default_rng(2)
    prompts = [rng.integers(0, workloads.QWEN3_VOCAB, n).astype(np.int32) for n in (1, 16, 35)]
    answers, steps = 3, 18  # past a page's end for each
    model = example.Decoder(w, theta, example.pages_needed(prompts, answers, steps))
    u = torch.rand(steps, 9, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    seen, plain_draw = [], zo.zo_draw

    def draw(logits, *args, **kw):
        seen.append((logits.clone(), kw))
        return plain_draw(logits, *args, **kw)

    monkeypatch.setattr(zo, "zo_draw", draw)
    tokens, logprobs = example.answer(model, prompts, answers, u, temperature=0.8, top_k=200, top_p=0.95)
    assert len(seen) == steps
    for a in range(9):
        prompt = torch.from_numpy(prompts[a // answers].astype(np.int64)).cuda()
        want = plain_logits(w, theta, torch.cat((prompt, tokens[a].long()[:-1])))[len(prompt) - 1:]
        got = torch.stack([s[0][a] for s in seen]).double()
        off = (got - want).square().mean(1).sqrt() / want.std(1)
        assert float(off.max()) <= 1 / 8, (a, off.tolist())
    for step in (0, 1, steps - 1):
        logits, kw = seen[step]
        assert logits.dtype == torch.bfloat16 and set(kw) == {"temperature", "top_k", "top_p", "logprobs"}
        host = logits.float().cpu().numpy()
        for a in range(9):
            token, lp = oracle.draw(host[a], float(u[step, a]), 0.8, 200, 0.95)
            assert int(tokens[a, step]) == token
            assert abs(float(logprobs[a, step]) - lp) <= 2.0 ** -22 * max(1.0, abs(lp))
