"""Decode-step operators on views that share a buffer without overlapping."""

import pytest
import torch

import paper_2609_38095_amd as zo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 7, 300])
def test_alternating_heads_in_place(tokens, dtype):
    """Queries and keys head by head in one tensor, rotated in place: as out of place, and what lies between them stays."""
    x = torch.randn(tokens, 4, 3, 64, generator=torch.Generator().manual_seed(tokens)).to("cuda", dtype)
    before = x.clone()
    q, k = x[:, :, 0], x[:, :, 1]
    positions, turns = torch.arange(tokens, dtype=torch.int32, device="cuda"), zo.zo_rotary_turns(64)
    gamma = torch.linspace(0.5, 1.5, 64, device="cuda").to(dtype)
    want = zo.zo_norm_rotate(q, k, positions, turns, q_gamma=gamma, k_gamma=gamma)
    zo.zo_norm_rotate(q, k, positions, turns, q_gamma=gamma, k_gamma=gamma, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, :, 2], before[:, :, 2])
