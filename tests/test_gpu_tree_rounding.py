"""Every form of the tree attention in bf16 is off by its output's own rounding, and not by that of the weights.

Tolerances, with e = 2^-24. Scores and sums are those of test_gpu_tree.py's bound(): 2 (dim + 8) e of the scores' magnitudes, keys / 8 + 64
steps of the weighted ones. A weight p in [2^n, 2^(n + 1)) is the sum of the largest bf16 below it and of what is left, at most 2^(n - 7), whose
own rounding to 8 bits is off by at most 2^(n - 16): 2^-16 p, 2^8 e. The output adds half a bf16 ulp. This holds whatever the rows of
the call are, so no case has another bound; what takes fp32 weights (heads, pages and strides of other kinds) has no 2^8 e."""

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
from oracle import tree as oracle
from test_gpu_tree import ATTEND, attend_case, bound, cache_of, dev, ints, near, normal, spoil, starts_of, trees, wide

pytestmark = pytest.mark.gpu


def steps_of(dim, keys, big, page, layout):
    """bound() of two-part weights, or of fp32 ones where a call takes them."""
    matrix = dim in (64, 128, 256) and page % 16 == 0 and layout != "odd"
    return bound(dim, keys, big, "bf16" if matrix else "f32")


@pytest.mark.parametrize("kind", ["chain", "tree"])
@pytest.mark.parametrize("case", ATTEND, ids=[str(i) for i in range(len(ATTEND))])
def test_outputs_are_off_by_their_own_rounding(case, kind):
    cached, counts, hq, hk, dim, page, layout, scale = case
    q, kc, vc, table, used = attend_case(cached, counts, hq, hk, dim, page, layout, "bf16")
    starts, scale, seen = starts_of(counts), dim ** -0.5 if scale is None else scale, None
    if kind == "tree":
        seen = oracle.lay(starts, cached, sum(counts), trees(counts, 5), max(1, -(-max(counts) // 64)))[3]
    want, _, mag, big = oracle.attend(wide(q), wide(kc), wide(vc), table, cached, starts, seen, scale)
    spoil(kc, vc, table, used, page)
    out = zo.zo_tree_attend(q, kc, vc, dev(table), ints(cached), dev(starts), None if seen is None else dev(seen), scale)
    near(out, want, mag, steps_of(dim, 3100, big, page, layout)[..., None], "bf16")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("counts", [[40] * 3, [300, 1], [3000]])
def test_rows_behind_a_long_context(counts, dim):
    """Sampled rows of chains behind up to 2,000 tokens, in calls of few and many rows."""
    cached, hq, hk, page = [2000 - 700 * s for s in range(len(counts))], 4, 2, 32
    width = -(-(max(counts) + 2000) // page)
    pages = len(counts) * width
    kc, vc = cache_of("tokens", 31, pages, hk, page, dim, "bf16")
    table = np.random.default_rng(3).permutation(pages).astype(np.int32).reshape(len(counts), width)
    starts = starts_of(counts)
    q = normal(4, (int(starts[-1]), hq, dim), "bf16", 1.5)
    out = zo.zo_tree_attend(q, kc, vc, dev(table), ints(cached), dev(starts))
    for s, n in enumerate(counts):
        k, v = (c[dev(table[s]).long()].transpose(0, 1).reshape(hk, -1, dim).double() for c in (kc, vc))
        for i in sorted({0, n // 3, n - 1}):
            live = cached[s] + i + 1
            for h in range(hq):
                row = q[int(starts[s]) + i, h].double()
                x = k[h // 2, :live] @ row * dim ** -0.5
                w = torch.softmax(x, 0)
                big = float((k[h // 2, :live].abs() @ row.abs()).max()) * dim ** -0.5
                near(out[int(starts[s]) + i, h], wide(w @ v[h // 2, :live]), wide(w @ v[h // 2, :live].abs()), bound(dim, live, big, "bf16"), "bf16")


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (256, 16)])
@pytest.mark.parametrize("nodes", [3, 64])
@pytest.mark.parametrize("rise", [0.25, -0.25, 1.0])
def test_weights_that_wait_while_the_bound_rises(dim, page, nodes, rise):
    """Scores that rise (or fall) with every key: both parts of the weights that wait are rescaled with the sums."""
    cached, counts = [180, 20], [nodes] * 2
    q, kc, vc, table, used = attend_case(cached, counts, 8, 2, dim, page, "heads", "bf16")
    q[..., 0] = 1.0
    kc *= 0.05
    for s, n in enumerate(used):
        for j in range(n):
            kc[int(table[s, j // page]), :, j % page, 0] = rise * j
    starts = starts_of(counts)
    want, _, mag, big = oracle.attend(wide(q), wide(kc), wide(vc), table, cached, starts, None, 0.4)
    spoil(kc, vc, table, used, page)
    out = zo.zo_tree_attend(q, kc, vc, dev(table), ints(cached), dev(starts), scale=0.4)
    near(out, want, mag, steps_of(dim, 250, big, page, "heads")[..., None], "bf16")


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (256, 16), (96, 16), (64, 5)])
@pytest.mark.parametrize("nodes", [3, 64])
def test_a_row_that_sees_one_key_has_its_value(dim, page, nodes):
    """(p v) / p is within 2^-15 of v, a bf16 number: it rounds to v."""
    q, kc, vc, table, _ = attend_case([0, 0], [nodes] * 2, 8, 2, dim, page, "heads", "bf16")
    which = np.random.default_rng(2).integers(0, nodes, 2 * nodes)
    seen = np.left_shift(np.uint64(1), which.astype(np.uint64)).view(np.int64)[:, None]
    out = zo.zo_tree_attend(q, kc, vc, dev(table), ints([0, 0]), ints([0, nodes, 2 * nodes]), dev(seen))
    for t, j in enumerate(which):
        v = vc[int(table[t // nodes, j // page]), :, j % page]
        assert torch.equal(out[t], v.repeat_interleave(4, 0))
