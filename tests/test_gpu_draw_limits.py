"""zo_draw at the ends of its logits' and temperatures' ranges, against the oracle: one workgroup for a row, and rows that are split."""

import math

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
from oracle import decode as oracle
from paper_2609_38095_amd import decode

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
SETTINGS = [  # temperature, top_k, top_p, min_p, u
    (1.0, 0, 1.0, 0.0, 0.4), (1.0, 0, 0.6, 0.0, 0.99), (1.0, 2, 1.0, 0.0, 0.7), (1e38, 0, 1.0, 0.0, 0.9), (1e38, 0, 0.5, 0.0, 0.3),
    (1e38, 3, 0.9, 0.0, 0.999), (3e37, 700, 0.9, 0.1, 0.6), (math.inf, 0, 1.0, 0.0, 0.77), (math.inf, 0, 0.3, 0.0, 0.5),
    (math.inf, 5, 0.9, 1.0, 0.99), (0.0, 0, 1.0, 0.0, 0.5), (1e-38, 0, 0.9, 0.0, 0.6)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [7, 1009, 16_400, 70_001])
@pytest.mark.parametrize("ends", ["both", "infinite", "finite"])
def test_the_largest_numbers(vocab, ends, dtype):
    """Rows that hold +inf, the largest finite number, or both, with NaN, -inf and the lowest number among ordinary logits."""
    most, rows = torch.finfo(dtype).max, len(SETTINGS)
    x = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(vocab)).mul_(2).to(dtype)
    at = [int(i * vocab / 7) for i in range(7)]
    x[:, at[0]], x[:, at[2]], x[:, at[3]], x[:, at[5]] = math.nan, -math.inf, -most, most / 2
    if ends != "infinite":
        x[:, at[4]] = most
    if ends != "finite":
        x[:, at[1]], x[:, at[6]] = math.inf, math.inf
    dev = x.cuda()
    t, k, p, m, u = (torch.tensor(c, dtype=torch.int32 if i == 1 else torch.float32, device="cuda") for i, c in enumerate(zip(*SETTINGS)))
    for with_k in (True, False):
        one = zo.zo_draw(dev, u, t, k if with_k else None, p, m, logprobs=True)
        assert (decode._lib().zo_draw_work(rows, vocab, with_k) > 0) == (vocab > (65_536 if with_k else 16_383))  # split
        many = zo.zo_draw(dev.repeat(4, 1), u.repeat(4), t.repeat(4), k.repeat(4) if with_k else None, p.repeat(4), m.repeat(4), logprobs=True)
        assert torch.equal(many[0], one[0].repeat(4)) and torch.equal(many[1], one[1].repeat(4))
        for b, (ti, ki, pi, mi, ui) in enumerate(SETTINGS):
            want, lp = oracle.draw(x[b].float().numpy(), ui, ti, ki if with_k else 0, pi, mi, most=most)
            assert int(one[0][b]) == want, (b, SETTINGS[b], with_k)
            assert float(one[1][b]) == lp or abs(float(one[1][b]) - lp) <= 4 * E * max(1.0, abs(lp)), (b, SETTINGS[b], with_k)


@pytest.mark.parametrize("top_p", [0.5, 0.95])
def test_weights_that_end_near_zero(top_p):
    """bf16 rows whose weights end at logits around 0: among those below 2^-10, in front of them and behind them."""
    low = [0.0, 5e-4, 2.0 ** -10, 0.00098, 2.0 ** -10 * (1 + 2.0 ** -7), 0.002, -0.00098, -0.002]
    t = torch.tensor([(16 - v) / 32 for v in low], device="cuda")  # 32 temperatures below the largest
    x = torch.randn(len(low), 9000, generator=torch.Generator().manual_seed(1)).mul_(4).clamp_(max=15.5)
    x[:, ::5] *= 2.0 ** -12
    x[:, ::7] = 0.0
    x[:, 77] = 16.0
    x = x.bfloat16()
    u = torch.linspace(0.05, 0.999, len(low), device="cuda")
    token, lp = zo.zo_draw(x.cuda(), u, t, top_p=torch.full((len(low),), top_p, device="cuda"), logprobs=True)
    for b in range(len(low)):
        want, exact = oracle.draw(x[b].float().numpy(), float(u[b]), float(t[b]), 0, top_p, most=torch.finfo(torch.bfloat16).max)
        assert int(token[b]) == want and abs(float(lp[b]) - exact) <= 4 * E * max(1.0, abs(exact)), (b, low[b])
