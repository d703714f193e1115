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
