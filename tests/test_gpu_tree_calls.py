"""Calls of the operators for several new tokens that are easy to forget, on the GPU."""

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
from oracle import tree as oracle
from test_gpu_tree import E, attend_case, cache_of, dev, ints, near, normal, starts_of, trees, wide

pytestmark = pytest.mark.gpu


# ---- moves

@pytest.mark.parametrize("layers", [1, 3, 150])
def test_keep_of_shared_caches(layers):
    """Layers that share a cache, and keys that are the values: each tensor's rows move once, in one launch or several."""
    kc, vc = cache_of("heads", 1, 12, 2, 4, 64, "bf16")
    table, lengths = np.arange(12, dtype=np.int32).reshape(3, 4), [0, 5, 2]
    path = np.array([[0, 2, 3, 5, 6], [1, 2, 4, 5, 7], [0, 1, 5, -1, -1]], np.int32)
    wants = [oracle.keep(wide(t), table, lengths, path) for t in (kc, vc)]
    for tensors in ((kc.clone(), vc.clone()), (kc.clone(), None)):
        k, v = tensors
        zo.zo_tree_keep([k] * layers, [k if v is None else v] * layers, dev(table), ints(lengths), dev(path))
        assert np.array_equal(wide(k), wants[0]) and (v is None or np.array_equal(wide(v), wants[1]))


# ---- put

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(128, 16), (20, 5)])
def test_a_token_without_a_position_is_not_put(dim, page, dtype):
    """Padding: a negative position, a negative place, or both; what is cached at the place stays."""
    n, hq, hk, width = 9, 4, 2, 3
    table = dev(np.arange(3 * width, dtype=np.int32).reshape(3, width))
    x = normal(1, (n, hq + 2 * hk, dim), dtype)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    kc, vc = cache_of("heads", 5, 3 * width, hk, page, dim, dtype)
    first = kc.clone(), vc.clone()
    seqs, places, positions = [0, 0, 0, 1, 1, 1, 2, 2, 2], [0, 1, -1, 3, 4, 5, -1, 7, 8], [0, -1, 2, 3, -2 ** 31, 4, -1, 7, -1]
    turns = zo.zo_rotary_turns(dim)
    zo.zo_norm_rotate_put(q, k, v, kc, vc, table, ints(positions), turns, seqs=ints(seqs), places=ints(places))
    ko = zo.zo_norm_rotate(None, k, ints(positions), turns)[1]
    for t in range(n):
        if places[t] >= 0 and positions[t] >= 0:
            at = int(table[seqs[t], places[t] // page]), slice(None), places[t] % page
            first[0][at], first[1][at] = ko[t], v[t]
    assert torch.equal(kc, first[0]) and torch.equal(vc, first[1])


# ---- walk

@pytest.mark.parametrize("kind", ["tree", "chain"])
@pytest.mark.parametrize("counts,words", [([100], 1), ([63, 64, 65, 200], 1), ([130, 1, 0, 700], 2), ([600, 512, 513], 8)])
def test_the_walk_ends_where_the_masks_do(counts, words, kind):
    """Every draw agrees: a walk goes on to the last token that zo_tree_lay gave a place, and what it moves was put."""
    n, starts = sum(counts), np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    parents = np.concatenate([np.arange(c) - 1 for c in counts]).astype(np.int32) if kind == "tree" else None
    drafted = np.arange(n, dtype=np.int32)
    args = dev(drafted), dev(drafted + 1), dev(starts)
    own = None if parents is None else dev(parents)
    lengths = ints([9] * len(counts))
    places = zo.zo_tree_lay(args[2], lengths, n, own, words)[2].cpu().numpy()
    path, tokens, walked = zo.zo_tree_accept(*args, 800, own, words=words)
    for g, w in zip((path, tokens, walked), oracle.accept(drafted, drafted + 1, starts, 800, parents, words)):
        assert np.array_equal(g.cpu().numpy(), w)
    assert walked.tolist() == [min(c, 64 * words) for c in counts]
    for s, c in enumerate(walked.tolist()):
        assert (places[starts[s] + path[s, :c].cpu().numpy()] >= 0).all()
    assert zo.zo_tree_accept(*args, 800, own)[2].tolist() == counts  # without words: chains of any length
    for wrong in (-1, 9):
        with pytest.raises(zo.ZoError):
            zo.zo_tree_accept(*args, 800, own, words=wrong)


# ---- attention

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 48), (256, 32), (96, 16)])
@pytest.mark.parametrize("nodes", [3, 70])
@pytest.mark.parametrize("score", [-3e38, 3e38, 7e9, -7e9, 2.0 ** 25 + 2.0 ** 18])
def test_scores_of_any_finite_size(score, nodes, dim, page, dtype):
    """Equal scores, one product each, so equal weights whatever a score's rounding: the mean of the values, and no score's own error. Every seventh
    key's is far below and has no part."""
    cached, counts, scale = [100, 0], [nodes] * 2, 0.2
    q, kc, vc, table, used = attend_case(cached, counts, 4, 2, dim, page, "heads", dtype)
    q.zero_(), kc.zero_()
    q[..., 0], kc[..., 0] = 1.0, score
    for s, n in enumerate(used):
        for j in range(6, n, 7):
            kc[int(table[s, j // page]), :, j % page, 0] = -abs(score) * 1.125
    starts = starts_of(counts)
    for seen in (None, oracle.lay(starts, cached, 2 * nodes, trees(counts, 3), 2)[3]):
        want, lse, mag, _ = oracle.attend(wide(q), wide(kc), wide(vc), table, cached, starts, seen, scale)
        out, sums = zo.zo_tree_attend(q, kc, vc, dev(table), ints(cached), dev(starts), None if seen is None else dev(seen), scale, lse=True)
        near(out, want, mag, 170 / 8 + 64 + (2.0 ** 8 if dtype == "bf16" else 0), dtype)
        # the score, times scale log2(e) and ln 2 in fp32, scale itself rounded: below 8 e
        assert np.all(np.abs(wide(sums) - lse) <= 8 * E * np.abs(lse) + 1e-5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 48), (256, 32), (96, 16)])
@pytest.mark.parametrize("nodes", [3, 70])
@pytest.mark.parametrize("scale", [0.0, 1e-40])
def test_scales_of_0_and_below_the_normal_ones(scale, nodes, dim, page, dtype):
    """Scores of single products up to 3e38 times a scale that is nothing, or next to it. The latter is a multiple of 2^-149, as its product with
    log2(e) is: scores of up to 0.04 are off by 2^-149 / 1e-40 of themselves, which moves a weight by 14 e at most, twice."""
    cached, counts = [100, 0], [nodes] * 2
    q, kc, vc, table, _ = attend_case(cached, counts, 4, 2, dim, page, "heads", dtype)
    q.zero_()
    q[..., 0] = 1.0
    kc[..., 0] = (kc[..., 0].clamp(-3, 3) * 1e38).to(kc.dtype)
    starts = starts_of(counts)
    want, lse, mag, _ = oracle.attend(wide(q), wide(kc), wide(vc), table, cached, starts, None, scale)
    out, sums = zo.zo_tree_attend(q, kc, vc, dev(table), ints(cached), dev(starts), scale=scale, lse=True)
    near(out, want, mag, 170 / 8 + 64 + 28 + (2.0 ** 8 if dtype == "bf16" else 0), dtype)
    assert np.all(np.abs(wide(sums) - lse) <= 8 * E * np.abs(lse) + 64 * E)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,nodes", [(64, 3), (64, 60), (128, 3), (128, 60), (256, 30), (40, 9)])
def test_queries_results_masks_and_tables_may_be_views(dim, nodes, dtype):
    """Rows that begin at any element, heads and tokens any distance apart, masks and a table of wider tensors: the bits of a call with tensors of
    their own, and nothing beside the result's rows is written."""
    cached, counts, hq, hk, page = [70, 200], [nodes, nodes + 1], 4, 2, 16
    q, kc, vc, table, _ = attend_case(cached, counts, hq, hk, dim, page, "heads", dtype)
    n, starts = sum(counts), dev(starts_of(counts))
    seen = dev(oracle.lay(starts_of(counts), cached, n, trees(counts, 3), 2)[3])
    lengths, own_table = ints(cached), dev(table)
    want, sums = zo.zo_tree_attend(q, kc, vc, own_table, lengths, starts, seen, lse=True)
    wide_q = torch.zeros(n, hq + 3, dim + 5, dtype=q.dtype, device="cuda")
    wide_q[:, 1:1 + hq, 3:3 + dim] = q
    wide_seen = torch.full((n, 5), -1, dtype=torch.int64, device="cuda")
    wide_seen[:, 2:4] = seen
    wide_table = torch.full((2, table.shape[1] + 7), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    wide_table[:, 3:3 + table.shape[1]] = own_table
    buffer = torch.full((hq + 1, n + 2, dim + 3), 7.0, dtype=q.dtype, device="cuda")
    out = buffer[:hq, 1:1 + n, 1:1 + dim].transpose(0, 1)
    got, got_sums = zo.zo_tree_attend(wide_q[:, 1:1 + hq, 3:3 + dim], kc, vc, wide_table[:, 3:3 + table.shape[1]], lengths, starts, wide_seen[:, 2:4],
                                      out=out, lse=True)
    assert got.data_ptr() == out.data_ptr() and torch.equal(out, want) and torch.equal(got_sums, sums)
    out.fill_(7.0)
    assert bool((buffer == 7.0).all())
