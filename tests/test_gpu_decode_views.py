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


def test_strides_of_single_entries_do_not_count():
    """A cache of one key head, its values made in another order of axes: the same places, whatever the head's stride says."""
    k = torch.randn(6, 1, 16, 64, device="cuda")
    v = torch.randn(6, 16, 1, 64, device="cuda").transpose(1, 2)
    assert k.stride() != v.stride()
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    q, at = torch.randn(2, 4, 64, device="cuda"), torch.tensor([20, 5], dtype=torch.int32, device="cuda")
    plain = v.contiguous().view(6, 1, 16, 64).clone()
    same = zo.zo_cache_attend(q, k, plain, table, at)
    assert plain.stride() == k.stride() and torch.equal(zo.zo_cache_attend(q, k, v, table, at), same)
    new = torch.randn(2, 1, 64, device="cuda")
    zo.zo_norm_rotate_put(None, new, new, k, v, table, at)
    assert torch.equal(k[1, :, 4], new[0]) and torch.equal(v[1, :, 4], new[0]) and torch.equal(v[2, :, 5], new[1])
    zo.zo_cache_copy([k], [v], [1], [5])
    assert torch.equal(k[5], k[1]) and torch.equal(v[5], v[1])
