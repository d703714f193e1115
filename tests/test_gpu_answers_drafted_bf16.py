"""Drafted answers as the example ships them, in bf16, with trees of many rows: each walked token is what a plain decoder's logits give.

Drafted and plain answers go through different products and attentions, so in bf16 their logits differ by roundings, and a draw that
these decide is another one; from there on the answers differ. What holds is that every answer is a right one: its logits are the plain decoder's behind
its own tokens. Tolerance as for single tokens (test_gpu_answers_cuts.py): some 30 tensors on the way are rounded to bf16, by at most 2^-9
of their values each; were all of it, doubled, to add up, it would be 64 2^-9 = 1/8 of the logits' spread."""

import numpy as np
import torch
import pytest

import paper_2609_38095_amd as zo
import workloads
from oracle import decode as oracle
from test_gpu_answers import example, plain_logits

pytestmark = pytest.mark.gpu


def test_drafted_bf16_answers_are_the_plain_decoders(monkeypatch):
    w = example.SMALL
    theta = torch.empty(w.n, dtype=torch.bfloat16, device="cuda")
    workloads.fill_model_buffer_device(theta, w)
    rng = np.random.default_rng(5)
    prompts = [rng.integers(0, workloads.QWEN3_VOCAB, n).astype(np.int32) for n in (1, 16, 35)]
    answers, steps, n = 3, 18, 9
    model = example.Decoder(w, theta, example.pages_needed(prompts, answers, steps) + n * 3)
    u = torch.rand(steps, n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    settings = dict(temperature=0.8, top_k=200, top_p=0.95)
    plain, _ = example.answer(model, prompts, answers, u, **settings)
    # six drafts that are right at every other place: with the plain answers as one more, trees of up to 29 tokens
    drafts = [plain]
    for _ in range(6):
        other = torch.from_numpy(rng.integers(0, workloads.QWEN3_VOCAB, (n, steps)).astype(np.int32)).cuda()
        other[:, ::2] = plain[:, ::2]
        drafts.append(other)

    draws, walks, rows = [], [], []
    plain_draw, plain_accept, plain_attend = zo.zo_draw, zo.zo_tree_accept, zo.zo_tree_attend

    def draw(logits, *args, **kw):
        draws.append((logits.clone(), args[0].clone()))
        return plain_draw(logits, *args, **kw)

    def accept(drafted, drawn, starts, *args, **kw):
        got = plain_accept(drafted, drawn, starts, *args, **kw)
        walks.append((starts.tolist(), got[0].tolist(), got[2].tolist()))
        return got

    def attend(q, k_cache, v_cache, table, *args, **kw):
        rows.append(q.shape[0] * q.shape[1] / k_cache.shape[1] / table.shape[0])
        return plain_attend(q, k_cache, v_cache, table, *args, **kw)

    monkeypatch.setattr(zo, "zo_draw", draw)
    monkeypatch.setattr(zo, "zo_tree_accept", accept)
    monkeypatch.setattr(zo, "zo_tree_attend", attend)
    tokens, logprobs, passes = example.answer_drafted(model, prompts, answers, u, drafts, **settings)
    assert tokens.shape == logprobs.shape == (n, steps) and len(draws) == len(walks) + 1 and max(rows) > 32
    # the logits behind each answer's tokens: its row of the first draw, then those of the walked paths
    behind = [[(draws[0][0][a], draws[0][1][a])] for a in range(n)]
    for (logits, numbers), (starts, path, walked) in zip(draws[1:], walks):
        live = [a for a in range(n) if len(behind[a]) < steps]
        assert len(live) == len(walked)
        for k, a in enumerate(live):
            behind[a] += [(logits[starts[k] + i], numbers[starts[k] + i]) for i in path[k][:walked[k]]]
    for a in range(n):
        prompt = torch.from_numpy(prompts[a // answers].astype(np.int64)).cuda()
        want = plain_logits(w, theta, torch.cat((prompt, tokens[a].long()[:-1])))[len(prompt) - 1:]
        got = torch.stack([x for x, _ in behind[a]]).double()
        off = (got - want).square().mean(1).sqrt() / want.std(1)
        assert float(off.max()) <= 1 / 8, (a, off.tolist())
        for step in (0, 1, 2, steps - 1):
            assert float(behind[a][step][1]) == float(u[step, a])
            token, lp = oracle.draw(behind[a][step][0].float().cpu().numpy(), float(u[step, a]), 0.8, 200, 0.95)
            assert int(tokens[a, step]) == token
            assert abs(float(logprobs[a, step]) - lp) <= 2.0 ** -22 * max(1.0, abs(lp))
