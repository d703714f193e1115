"""The operators for several new tokens of a sequence on the GPU, against the oracle in 64 bits.

Tolerances follow from the arithmetic, with e = 2^-24 (half an fp32 ulp, relative). A score is a sum of dim products and one scaling, off
by at most (dim + 8) e of its products' magnitudes, which moves each weight by that share, twice (weight and sum). The
weighted sum adds a rounding for each 16 keys and each of a bf16 weight's two parts, a rescaling and a join now and
then: below keys / 8 + 64. bf16 weights are two parts of 8 bits each (2^-16 of the weight, 2^8 e); with more than 32 rows (a new
token and a query head of a key head's) a sequence, and heads of 64 or 128, they are rounded once behind their sum: with w' = w (1 + d),
|d| <= 2^-8, sum w' v / sum w - sum w v / sum w is below 2^-8 of the weighted magnitudes, 2^16 e; the log-sum knows nothing of that. A
bf16 output adds half a bf16 ulp. Whole numbers and moved rows are equal.
"""

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
from oracle import tree as oracle

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def wide(t):
    return t.detach().double().cpu().numpy()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(a):
    return dev(np.array(a, np.int32))


def normal(seed, shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(0, scale, generator=g).to(TYPES[dtype])


def near(got, want, magnitude, steps, dtype):
    got = wide(got)
    assert np.array_equal(np.isfinite(got), np.isfinite(want))
    fine = np.isfinite(want)
    half_ulp = np.exp2(np.floor(np.log2(np.maximum(np.abs(np.where(fine, want, 1.0)), 1e-38))) - 8)
    most = steps * E * magnitude + (half_ulp if dtype == "bf16" else 0.0) + 1e-37
    worst = np.max(np.where(fine, np.abs(np.where(fine, got - want, 0.0)) / most, 0.0)) if got.size else 0.0
    assert worst <= 1.0, f"off by {worst:.2f} of what rounding allows"


def bound(dim, keys, big, dtype, rows=0):
    """Steps of rounding behind an output, relative to the weighted magnitudes of the values. rows: of a sequence, on average (0: behind a
    log-sum, whose weights are not rounded to bf16)."""
    once = rows > 32 and dim in (64, 128)
    return 2 * (dim + 8) * big + keys / 8 + 64 + (0 if dtype == "f32" else 2.0 ** 16 if once else 2.0 ** 8)


def trees(counts, seed, roots=0.05):
    """Random trees: half of the tokens go on from the one before, a few come behind the cached tokens too."""
    rng = np.random.default_rng(seed)
    got = []
    for n in counts:
        for i in range(n):
            got.append(-1 if i == 0 or rng.random() < roots else i - 1 if rng.random() < 0.5 else int(rng.integers(i)))
    return np.array(got, np.int32)


def starts_of(counts):
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int32)


# ---- layout

LAY = [
    # counts, words, rows in front, rows behind
    ([1], 1, 0, 0), ([0, 3, 0], 1, 2, 3), ([64], 1, 0, 0), ([65, 1, 64, 63], 2, 0, 5), ([512, 7], 8, 0, 0), ([200] * 40, 4, 1, 0),
    ([70, 10], 1, 0, 0), ([600], 8, 0, 0), ([130, 129], 3, 0, 0), ([], 1, 0, 4),
]


@pytest.mark.parametrize("case", LAY, ids=[str(i) for i in range(len(LAY))])
@pytest.mark.parametrize("kind", ["tree", "chain", "chain with masks"])
def test_lay(case, kind):
    counts, words, front, behind = case
    starts = starts_of(counts) + front
    tokens = int(starts[-1]) + behind
    parents = np.concatenate((np.full(front, 5, np.int32), trees(counts, tokens), np.full(behind, 2, np.int32))) if kind == "tree" else None
    lengths = np.random.default_rng(1).integers(-3, 5000, len(counts)).astype(np.int32)
    if counts:
        lengths[0] = 2 ** 31 - 3  # sums saturate
    words = 0 if kind == "chain" else words
    got = zo.zo_tree_lay(dev(starts), dev(lengths), tokens, None if parents is None else dev(parents), words)
    want = oracle.lay(starts, lengths, tokens, parents, words)
    for g, w in zip(got, want):
        assert (g is None) == (w is None)
        assert g is None or np.array_equal(g.cpu().numpy(), w)


def test_lay_has_room_for_any_tree_by_default():
    n, parents = 300, trees([300], 2)
    got = zo.zo_tree_lay(ints([0, n]), ints([9]), n, dev(parents))
    for g, w in zip(got, oracle.lay(np.array([0, n]), [9], n, parents, 5)):
        assert np.array_equal(g.cpu().numpy(), w)
    assert zo.zo_tree_lay(ints([0, 0]), ints([9]), 0, ints([]))[3].shape == (0, 1)


def test_lay_takes_any_parents():
    """Parents that are not below their token, or negative, count as none; so the masks are those of the trees without them."""
    rng = np.random.default_rng(4)
    counts = [100, 30, 64]
    n = sum(counts)
    parents = np.concatenate([rng.integers(-5, c + 5, c) for c in counts]).astype(np.int32)
    parents[[3, 40]] = [2 ** 31 - 1, -2 ** 31]
    got = zo.zo_tree_lay(ints(starts_of(counts)), ints([0, 9, 100]), n, dev(parents), 2)
    want = oracle.lay(starts_of(counts), [0, 9, 100], n, parents, 2)
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)


# ---- put

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,rotary,page", [(128, 128, 16), (64, 32, 5), (20, 20, 7)])
def test_put_at_places(dim, rotary, page, dtype):
    """Turned by the positions, put at the places: as zo_norm_rotate and a plain assignment."""
    counts, lengths = [5, 1, 9, 3], [3, 0, 17, 30]
    starts, n = starts_of(counts), sum(counts)
    seq_of, positions, places, _ = zo.zo_tree_lay(dev(starts), ints(lengths), n, dev(trees(counts, 2)))
    width, hq, hk = 8, 4, 2
    table = np.random.default_rng(0).permutation(4 * width).astype(np.int32).reshape(4, width)
    table[2, 17 // page] = -1
    x = normal(1, (n, hq + 2 * hk, dim), dtype)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    kc, vc = (normal(5 + i, (4 * width, hk, page, dim), dtype) for i in range(2))
    want = kc.clone(), vc.clone()
    turns, gamma = zo.zo_rotary_turns(rotary), 1 + normal(3, (dim,), dtype, 0.1)
    places[4] = -1  # not put; its query is turned all the same
    got = zo.zo_norm_rotate_put(q, k, v, kc, vc, dev(table), positions, turns, q_gamma=gamma, k_gamma=gamma, seqs=seq_of, places=places)
    qo, ko = zo.zo_norm_rotate(q, k, positions, turns, q_gamma=gamma, k_gamma=gamma)
    assert torch.equal(got, qo)
    for t, (s, at) in enumerate(zip(seq_of.tolist(), places.tolist())):
        if at >= 0 and at // page < width and table[s, at // page] >= 0:
            want[0][table[s, at // page], :, at % page] = ko[t]
            want[1][table[s, at // page], :, at % page] = v[t]
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


# ---- attention

ATTEND = [
    # cached, new tokens, q heads, k heads, dim, page, layout, scale
    ([0], [1], 1, 1, 64, 16, "heads", None),
    ([0, 5, 0], [1, 0, 3], 4, 2, 64, 16, "heads", None),
    ([31, 32, 33, 127, 128, 129, 0], [1, 2, 1, 3, 1, 2, 4], 4, 4, 128, 16, "tokens", None),
    ([100, 3, 700], [7, 8, 5], 8, 2, 128, 16, "heads", None),
    ([1037], [12], 32, 8, 128, 16, "heads", None),
    ([60, 500, 0, 64], [64, 33, 20, 1], 12, 3, 64, 32, "tokens", None),
    ([3000, 10], [20, 64], 16, 8, 128, 64, "both", None),
    ([200, 77], [100, 130], 6, 2, 128, 48, "heads", 0.3),
    ([70, 20], [30, 9], 24, 1, 64, 16, "odd", None),
    ([40, 300], [40, 3], 4, 2, 256, 16, "heads", None),
    ([40, 300], [2, 3], 4, 2, 256, 16, "both", None),
    ([50, 9], [12, 40], 6, 2, 80, 24, "odd", None),
    ([50, 9], [2, 4], 3, 1, 20, 1, "heads", None),
    ([70, 20, 3], [3, 2, 50], 4, 2, 1, 3, "heads", 1.0),
    ([90, 5], [33, 70], 2, 1, 200, 24, "tokens", None),
    ([120, 64], [20, 3], 4, 2, 128, 16, "heads", 0.0),
    ([120, 64], [20, 3], 4, 2, 64, 16, "heads", -0.2),
    ([400, -3, 10 ** 9, 395], [10, 40, 3, 20], 4, 2, 128, 64, "heads", 2.0),
]


def cache_of(kind, seed, pages, heads, page, dim, dtype):
    if kind == "heads":
        return [normal(seed + i, (pages, heads, page, dim), dtype) for i in range(2)]
    if kind == "tokens":
        return [normal(seed + i, (pages, page, heads, dim), dtype).transpose(1, 2) for i in range(2)]
    if kind == "both":  # keys and values in one tensor
        x = normal(seed, (pages, 2, heads, page, dim), dtype)
        return [x[:, 0], x[:, 1]]
    x = normal(seed, (pages, 2, page, heads, dim + 3), dtype)[..., 1:1 + dim].transpose(2, 3)
    return [x[:, 0], x[:, 1]]


def spoil(kc, vc, table, used, page):
    """What lies behind the ends, and in pages of no one, is infinite or not a number."""
    for s, n in enumerate(used):
        n = min(n, table.shape[1] * page)
        if n % page and 0 <= table[s, n // page] < len(kc):
            kc[table[s, n // page], :, n % page:] = float("nan")
            vc[table[s, n // page], :, n % page:] = float("inf")
    held = {int(p) for s, n in enumerate(used) for p in table[s, :-(-min(n, table.shape[1] * page) // page)]}
    for p in set(range(len(kc))) - held:
        kc[p], vc[p] = float("inf"), float("nan")


def attend_case(cached, counts, hq, hk, dim, page, layout, dtype, room=400):
    """q, caches, table, and the lengths that the table holds."""
    used = [max(c, 0) + n for c, n in zip(cached, counts)]
    width = max(1, max(-(-min(u, max(room, 3100)) // page) for u in used))
    if max(used) > 10 ** 6:
        width = -(-room // page)
    pages = len(cached) * width + 3
    table = np.random.default_rng(7).permutation(pages)[:len(cached) * width].astype(np.int32).reshape(len(cached), width)
    kc, vc = cache_of(layout, 21, pages, hk, page, dim, dtype)
    q = normal(3, (sum(counts), hq, dim), dtype, 1.5)
    return q, kc, vc, table, used


def check(got, sums, want, dim, keys, dtype, rows):
    out, lse, mag, big = want
    there = ~np.isnan(lse)
    steps = bound(dim, keys, big, dtype, rows)
    near(got[dev(there)], out[there].reshape(-1, dim), mag[there].reshape(-1, dim), steps[there].reshape(-1, 1), dtype)
    sums = wide(sums)
    assert np.array_equal(np.isneginf(sums[there]), np.isneginf(lse[there]))
    fine = np.isfinite(lse)
    steps = bound(dim, keys, big, dtype)
    assert np.all(np.abs(sums[fine] - lse[fine]) <= (steps[fine] + 8 * np.abs(lse[fine])) * E)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["chain", "tree", "masks"])
@pytest.mark.parametrize("case", ATTEND, ids=[str(i) for i in range(len(ATTEND))])
def test_attend(case, kind, dtype):
    cached, counts, hq, hk, dim, page, layout, scale = case
    q, kc, vc, table, used = attend_case(cached, counts, hq, hk, dim, page, layout, dtype)
    n, words = sum(counts), max(1, -(-max(counts) // 64))
    starts = starts_of(counts)
    scale = dim ** -0.5 if scale is None else scale
    seen = None
    if kind == "tree":
        seen = oracle.lay(starts, cached, n, trees(counts, 5), words)[3]
    elif kind == "masks":  # any set of the new tokens, later ones and none at all among them
        rng = np.random.default_rng(9)
        seen = rng.integers(-2 ** 63, 2 ** 63, (n, words), dtype=np.int64)
        seen[rng.random(n) < 0.2] = 0
    want = oracle.attend(wide(q), wide(kc), wide(vc), table, cached, starts, seen, scale)
    spoil(kc, vc, table, used, page)
    args = (q, kc, vc, dev(table), ints(cached), dev(starts), None if seen is None else dev(seen), scale)
    out, sums = zo.zo_tree_attend(*args, lse=True)
    check(out, sums, want, dim, 3100, dtype, n * hq / hk / len(counts))
    assert torch.equal(out, zo.zo_tree_attend(*args))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs", [257, 1000])
def test_attend_many_sequences(seqs, dtype):
    """More sequences than a workgroup has threads; some without new tokens, one with many."""
    rng = np.random.default_rng(seqs)
    counts = rng.integers(0, 4, seqs)
    counts[seqs // 2] = 300
    cached = rng.integers(0, 60, seqs)
    q, kc, vc, table, used = attend_case(cached.tolist(), counts.tolist(), 4, 2, 64, 16, "heads", dtype)
    starts = starts_of(counts)
    want = oracle.attend(wide(q), wide(kc), wide(vc), table, cached, starts, None, 0.125)
    spoil(kc, vc, table, used, 16)
    out, sums = zo.zo_tree_attend(q, kc, vc, dev(table), dev(cached.astype(np.int32)), dev(starts), lse=True)
    check(out, sums, want, 64, 360, dtype, counts.sum() * 2 / seqs)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,dim,nodes", [(16, 64, 3), (32, 128, 40), (5, 64, 40), (5, 64, 3)])
def test_attend_absent_pages(page, dim, nodes, dtype):
    """Ids outside the cache leave their tokens out; a row that sees nothing else is empty."""
    cached, counts, width, pages = [8 * page, 3 * page + 2, 2 * page, 0], [nodes] * 4, 20, 100
    table = np.random.default_rng(8).permutation(pages)[:4 * width].astype(np.int32).reshape(4, width)
    for s, j, what in [(0, 0, -1), (0, 3, pages), (0, 4, 2 ** 31 - 1), (0, 7, -2 ** 31), (1, 3, -7), (3, 0, -1)]:
        table[s, j] = what
    table[2] = -1
    kc, vc = cache_of("heads", 2, pages, 2, page, dim, dtype)
    q, starts = normal(3, (4 * nodes, 4, dim), dtype), starts_of(counts)
    want = oracle.attend(wide(q), wide(kc), wide(vc), table, cached, starts, None, 0.2)
    spoil(kc, vc, table, [0 if s == 2 else c + n for s, (c, n) in enumerate(zip(cached, counts))], page)
    out, sums = zo.zo_tree_attend(q, kc, vc, dev(table), ints(cached), dev(starts), scale=0.2, lse=True)
    check(out, sums, want, dim, 400, dtype, 2 * nodes)
    assert not out[2 * nodes:3 * nodes].any() and bool(torch.isneginf(sums[2 * nodes:3 * nodes]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page,nodes", [(64, 16, 4), (64, 16, 60), (128, 16, 4), (128, 48, 60), (256, 32, 30), (20, 5, 40), (96, 16, 5)])
def test_values_reach_the_rows_that_see_them(dim, page, nodes, dtype):
    """Infinite and NaN keys and values of new tokens: rows that do not see them are as without them, rows that do have the infinity
    (or a NaN); of cached tokens: every row has it."""
    inf, nan = float("inf"), float("nan")
    cached, counts, hq, hk = [37, 3], [nodes, nodes], 8, 2
    q, kc, vc, table, _ = attend_case(cached, counts, hq, hk, dim, page, "heads", dtype)
    starts = starts_of(counts)
    parents = trees(counts, 3)
    seen = oracle.lay(starts, cached, 2 * nodes, parents, 1)[3]
    dt, dl, ds = dev(table), ints(cached), dev(starts)
    for masks in (None, dev(seen)):
        plain = zo.zo_tree_attend(q, kc, vc, dt, dl, ds, masks)
        k, v = kc.clone(), vc.clone()
        at = lambda s, j: (int(table[s, j // page]), slice(None), j % page)  # noqa: E731
        bad = {0: nodes // 2, 1: nodes - 1}
        for s, i in bad.items():
            v[at(s, cached[s] + i)][..., 3] = inf
            v[at(s, cached[s] + i)][..., 4] = nan
        v[at(0, 2)][..., 5] = -inf
        out = zo.zo_tree_attend(q, k, v, dt, dl, ds, masks)
        for s in (0, 1):
            for i in range(nodes):
                row, t = out[s * nodes + i], s * nodes + i
                sees = bad[s] <= i if masks is None else bool(int(seen[t, 0]) >> bad[s] & 1)
                if sees:
                    assert bool((row[:, 3] == inf).all()) and bool(row[:, 4].isnan().all())
                if s == 0:
                    assert bool((row[:, 5] == -inf).all())
                rest = [d for d in range(dim) if not (d in (3, 4) and sees or d == 5 and s == 0)]
                assert bool(torch.isfinite(row[:, rest]).all())
                # where a value is added by itself the sum has another order, and its weight is not rounded to bf16: off by 2^-8 of values
                # below 5 at the most, and by both results' rounding
                assert float((row[:, rest].float() - plain[t][:, rest].float()).abs().max()) <= (0.04 if dtype == "bf16" else 1e-4)
        # a key that is not a number: its own rows alone
        k[at(0, cached[0] + bad[0])][..., 0] = nan
        out = zo.zo_tree_attend(q, k, vc, dt, dl, ds, masks)
        for i in range(nodes):
            sees = bad[0] <= i if masks is None else bool(int(seen[i, 0]) >> bad[0] & 1)
            assert bool(out[i].isnan().all()) if sees else torch.equal(out[i], plain[i])
        assert torch.equal(out[nodes:], plain[nodes:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 48), (256, 32), (20, 5)])
@pytest.mark.parametrize("nodes", [3, 70])
def test_the_largest_finite_values_stay_finite(dim, page, nodes, dtype):
    """Weights are at most 1 while they are summed. The last cached score is 5.375 above the first (2^7.75), the others far below."""
    most = torch.finfo(TYPES[dtype]).max
    q, kc, vc, table, _ = attend_case([70, 130], [nodes] * 2, 4, 2, dim, page, "heads", dtype)
    kc.zero_(), vc.zero_(), q.zero_()
    q[..., 0] = 1.0
    kc[..., 0] = -40.0
    for s, n in ((0, 70), (1, 130)):
        kc[int(table[s, 0]), :, 0, 0] = 0.0
        kc[int(table[s, (n - 1) // page]), :, (n - 1) % page, 0] = 5.375
        vc[int(table[s, (n - 1) // page]), :, (n - 1) % page] = most
    out = zo.zo_tree_attend(q, kc, vc, dev(table), ints([70, 130]), dev(starts_of([nodes] * 2)), scale=1.0).float()
    assert bool(((out > 0.99 * most) & (out < most)).all())


@pytest.mark.parametrize("dim,group", [(64, 1), (64, 16), (128, 2), (256, 2), (96, 2)])
def test_means_of_the_largest_values_stay_finite(dim, group):
    """Every value the largest bf16 one: so is every mean, whatever the weights round to (2^-8 of it below at most, and its own rounding).
    Not so in fp32: a mean is off by a few e there, and the largest fp32 number times 1 + e is infinite."""
    most = torch.finfo(torch.bfloat16).max
    q, kc, vc, table, _ = attend_case([0, 200], [90, 70], 2 * group, 2, dim, 16, "heads", "bf16")
    vc.fill_(most)
    vc[..., 1::2] = -most
    for starts in ([0, 90, 160], [0, 1, 160]):
        out = zo.zo_tree_attend(q, kc, vc, dev(table), ints([0, 200]), ints(starts)).float()
        assert bool(((out.abs() <= most) & (out.abs() >= most * (1 - 2.0 ** -7))).all()) and bool((out[..., 0] > 0).all())


def test_attend_leaves_other_rows():
    """Rows in front of the first sequence's and behind the last one's stay as they were; starts outside the rows count as the
    nearest; the result may be a view."""
    kc, vc = cache_of("heads", 1, 20, 2, 16, 128, "bf16")
    q = normal(2, (12, 4, 128), "bf16")
    table = dev(np.arange(20, dtype=np.int32).reshape(4, 5))
    lengths = ints([5, 17, 0, 33])
    for starts in ([2, 4, 4, 7, 9], [-5, 4, 4, 7, 9], [3, 3, 3, 3, 10 ** 9], [0, 5, 10 ** 9, 10 ** 9, 10 ** 9]):
        buffer = torch.full((12, 2, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        out = buffer[:, 1]
        zo.zo_tree_attend(q, kc, vc, table, lengths, ints(starts), out=out)
        want = oracle.attend(wide(q), wide(kc), wide(vc), table.cpu().numpy(), [5, 17, 0, 33], starts, None, 128 ** -0.5)
        there = ~np.isnan(want[1][:, 0])
        assert torch.equal(out[dev(~there)], torch.full_like(out[dev(~there)], 7.0)) and bool((buffer[:, 0] == 7.0).all())
        steps = bound(128, 50, want[3], "bf16", 12 * 2 / 4)
        near(out[dev(there)], want[0][there], want[2][there], steps[there][..., None], "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_new_token_is_the_single_tokens_attention(dtype):
    """A chain of one is zo_cache_attend of one token more, up to the rounding of both."""
    cached = [0, 15, 16, 300, 1000]
    q, kc, vc, table, _ = attend_case(cached, [1] * 5, 16, 4, 128, 16, "heads", dtype)
    got = zo.zo_tree_attend(q, kc, vc, dev(table), ints(cached), ints(range(6)))
    want = zo.zo_cache_attend(q, kc, vc, dev(table), ints([c + 1 for c in cached]))
    assert float((got.float() - want.float()).abs().max()) <= (2.0 ** -7 if dtype == "bf16" else 2e-5)


@pytest.mark.parametrize("dim", [64, 128])
def test_attend_long_prompt(dim):
    """A chain of thousands behind a cached prefix: sampled rows against float64."""
    n, cached, hq, hk, page = 5001, 1030, 4, 2, 64
    q, kc, vc, table, used = attend_case([cached, 3], [n, 40], hq, hk, dim, page, "heads", "bf16", room=7000)
    width = -(-(n + cached) // page)
    table = np.random.default_rng(1).permutation(2 * width).astype(np.int32).reshape(2, width)
    kc, vc = cache_of("heads", 21, 2 * width, hk, page, dim, "bf16")
    out, sums = zo.zo_tree_attend(q, kc, vc, dev(table), ints([cached, 3]), ints([0, n, n + 40]), lse=True)
    k, v = (c[dev(table[0]).long()].transpose(0, 1).reshape(hk, -1, dim).double() for c in (kc, vc))
    for i in (0, 1, 63, 64, 1000, 2047, 3333, n - 1):
        for h in range(hq):
            live = cached + i + 1
            x = k[h // 2, :live] @ q[i, h].double() * dim ** -0.5
            w = torch.softmax(x, 0)
            want, mag = w @ v[h // 2, :live], w @ v[h // 2, :live].abs()
            big = float((k[h // 2, :live].abs() @ q[i, h].double().abs()).max()) * dim ** -0.5
            near(out[i, h], wide(want), wide(mag), bound(dim, live, big, "bf16", n), "bf16")
            assert abs(float(sums[i, h]) - float(torch.logsumexp(x, 0))) <= bound(dim, live, big, "bf16") * E + 1e-5


def test_attend_far_pages():
    """Offsets that pass 2^31 elements."""
    pages, heads, page, dim = 70_000, 16, 16, 128
    c = torch.empty(pages, heads, page, dim, dtype=torch.bfloat16, device="cuda")
    ids = [69_999, 66_000, 12, 65_536]
    for i, p in enumerate(ids):
        c[p] = normal(i, (heads, page, dim), "bf16")
    small = torch.stack([c[p] for p in ids])
    for nodes in (2, 50):
        q = normal(9, (nodes, heads, dim), "bf16")
        far = zo.zo_tree_attend(q, c, c, ints([ids]), ints([64 - nodes]), ints([0, nodes]))
        assert torch.equal(far, zo.zo_tree_attend(q, small, small, ints([range(4)]), ints([64 - nodes]), ints([0, nodes])))


# ---- walk

@pytest.mark.parametrize("kind", ["tree", "chain"])
@pytest.mark.parametrize("counts,most", [([1], 1), ([12, 0, 5, 30], 8), ([200, 1, 64], 24), ([3000, 1025, 1024, 2], 4000), ([50] * 300, 5)])
def test_accept(counts, most, kind):
    rng = np.random.default_rng(len(counts) + most)
    n, starts = sum(counts), starts_of(counts) + 2
    parents = np.concatenate((np.full(2, -1, np.int32), trees(counts, 1), np.full(3, 1, np.int32)))
    drafted, drawn = (rng.integers(0, 3 if kind == "tree" else 40, n + 5).astype(np.int32) for _ in range(2))
    for first, count in oracle.spans(starts, n + 5):  # draws mostly agree with a token behind
        for i in range(1, count):
            p = i - 1 if kind == "chain" else parents[first + i]
            if p >= 0 and rng.random() < 0.97:
                drawn[first + p] = drafted[first + i]
    own = parents if kind == "tree" else None
    got = zo.zo_tree_accept(dev(drafted), dev(drawn), dev(starts), most, None if own is None else dev(own))
    for g, w in zip(got, oracle.accept(drafted, drawn, starts, most, own)):
        assert np.array_equal(g.cpu().numpy(), w)


def test_accept_takes_the_first_of_equal_tokens():
    parents, drafted, drawn = [-1, 0, 0, 0, 2, 2, 3, 9], [5, 7, 8, 8, 1, 1, 1, 8], [8, 0, 1, 1, 2, 2, 2, 2]
    path, tokens, counts = zo.zo_tree_accept(ints(drafted), ints(drawn), ints([0, 8]), 5, ints(parents))
    assert path.tolist() == [[0, 2, 4, -1, -1]] and tokens.tolist() == [[8, 1, 2, -1, -1]] and counts.tolist() == [3]


@pytest.mark.parametrize("parents", [None, [-1, 0, 1, 1, 3]])
def test_accept_takes_no_negative_token(parents):
    """Places of a padded tree, behind a row that zo_draw found no token for."""
    drafted, drawn = [5, 7, -1, -1, -1], [7, -1, -1, -1, -1]
    got = zo.zo_tree_accept(ints(drafted), ints(drawn), ints([0, 5]), 5, None if parents is None else ints(parents))
    assert [g.tolist() for g in got] == [[[0, 1, -1, -1, -1]], [[7, -1, -1, -1, -1]], [2]]


def test_accept_walks_over_windows():
    """Branches whose tokens lie thousands of indices apart: a child behind the window of its parent."""
    n = 5000
    parents = np.full(n, -1, np.int32)
    walk = [0, 3, 900, 1023, 1024, 2500, 2501, 4999]
    drafted, drawn = np.full(n, 1, np.int32), np.full(n, 2, np.int32)
    for a, b in zip(walk, walk[1:]):
        parents[b], drafted[b], drawn[a] = a, 100 + b, 100 + b
    parents[4998], drafted[4998] = 3, 100 + 900  # a later sibling of the same token
    for most in (3, 20):
        path, tokens, counts = zo.zo_tree_accept(dev(drafted), dev(drawn), ints([0, n]), most, dev(parents))
        assert path[0, :counts[0]].tolist() == walk[:most] and counts.tolist() == [min(most, len(walk))]
        assert np.array_equal(path.cpu().numpy(), oracle.accept(drafted, drawn, [0, n], most, parents)[0])


# ---- moves

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layers,heads,dim,page,layout,most", [(1, 1, 64, 16, "heads", 4), (3, 8, 128, 16, "tokens", 16), (2, 2, 20, 5, "both", 9),
                                                               (60, 2, 8, 3, "heads", 7), (1, 3, 33, 1, "odd", 100), (2, 4, 64, 32, "both", 200)])
def test_keep(layers, heads, dim, page, layout, most, dtype):
    rng = np.random.default_rng(most)
    seqs, nodes = 7, most + 40
    lengths = np.array([0, 1, page - 1, page, 3 * page + 2, -4, 5], np.int32)
    width = -(-(max(lengths.max(), 0) + nodes) // page)
    pages = seqs * width + 2
    table = rng.permutation(pages)[:seqs * width].astype(np.int32).reshape(seqs, width)
    table[3, min(2, width - 1)], table[4, 3] = -1, pages
    path = np.full((seqs, most), -1, np.int32)
    for s in range(seqs):
        n = [most, 1, most // 2 + 1, most, most, most, 0][s]
        path[s, :n] = np.sort(rng.permutation(nodes - 1)[:n] + 1) if s != 1 else 0
        if s in (0, 3) and n:
            path[s, 0] = 0
    path[5, most // 2] = path[5, 0] if most > 2 else -1  # the walk ends where it does not rise
    path[2, most // 2 + 1:] = 3 + nodes
    path[2, min(most // 2 + 1, most - 1)] = -9  # and at a negative entry, whatever is behind it
    caches = [cache_of(layout, 10 * i, pages, heads, page, dim, dtype) for i in range(layers)]
    wants = [[oracle.keep(wide(t), table, lengths, path) for t in c] for c in caches]
    zo.zo_tree_keep([c[0] for c in caches], [c[1] for c in caches], dev(table), dev(lengths), dev(path))
    for c, w in zip(caches, wants):
        for t, x in zip(c, w):
            assert np.array_equal(wide(t), x)


def test_keep_behind_the_table():
    """Rows behind the table's end are neither read nor written; a path of a wider tensor."""
    kc, vc = cache_of("heads", 1, 4, 2, 4, 64, "f32")
    table = np.array([[0, 1], [2, 3]], np.int32)
    wide_path = np.array([[9, 2, 5, 7, 8, 9], [9, 1, 3, 2 ** 31 - 1, 0, 0]], np.int32)
    path = dev(wide_path)[:, 1:]
    wants = [oracle.keep(wide(t), table, [2, 2 ** 31 - 1], wide_path[:, 1:]) for t in (kc, vc)]
    zo.zo_tree_keep([kc], [vc], dev(table), ints([2, 2 ** 31 - 1]), path)
    assert np.array_equal(wide(kc), wants[0]) and np.array_equal(wide(vc), wants[1])


# ---- together

def step_tensors(dtype, seed=0):
    counts, cached = [6, 1, 9, 4], [10, 33, 0, 47]
    n, hq, hk, dim, page, width = sum(counts), 8, 2, 64, 16, 4
    x = normal(seed, (n, hq + 2 * hk, dim), dtype)
    kc, vc = cache_of("heads", seed + 1, 4 * width, hk, page, dim, dtype)
    table = dev(np.random.default_rng(seed).permutation(4 * width).astype(np.int32).reshape(4, width))
    return dict(q=x[:, :hq], k=x[:, hq:hq + hk], v=x[:, hq + hk:], kc=kc, vc=vc, table=table, starts=dev(starts_of(counts)),
                lengths=ints(cached), parents=dev(trees(counts, 1, 0.0)), n=n, drafted=ints(np.arange(n) % 3),
                logits=normal(seed + 5, (n, 3), "f32"), u=torch.linspace(0, 0.99, n, device="cuda"), turns=zo.zo_rotary_turns(dim))


def draft_step(s, stream=None):
    """A decode step of drafted trees: layout, put, attention, a draw behind each token, the walk, its moves."""
    seq_of, positions, places, seen = zo.zo_tree_lay(s["starts"], s["lengths"], s["n"], s["parents"], stream=stream)
    q = zo.zo_norm_rotate_put(s["q"], s["k"], s["v"], s["kc"], s["vc"], s["table"], positions, s["turns"], seqs=seq_of, places=places, stream=stream)
    out = zo.zo_tree_attend(q, s["kc"], s["vc"], s["table"], s["lengths"], s["starts"], seen, stream=stream)
    drawn = zo.zo_draw(s["logits"], s["u"], stream=stream)
    path, tokens, counts = zo.zo_tree_accept(s["drafted"], drawn, s["starts"], 6, s["parents"], stream=stream)
    zo.zo_tree_keep([s["kc"]], [s["vc"]], s["table"], s["lengths"], path, stream=stream)
    return out, path, tokens, counts


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_step_on_a_stream_and_in_a_graph(dtype):
    """The operators together: on another stream, and captured; every replay gives the eager step's bits, with other work between."""
    s = step_tensors(dtype)
    first = s["kc"].clone(), s["vc"].clone()
    want = draft_step(s)
    after = s["kc"].clone(), s["vc"].clone()
    assert int(want[3].min()) >= 1 and int(want[3].max()) > 1

    def reset():
        s["kc"].copy_(first[0]), s["vc"].copy_(first[1])
        torch.cuda.synchronize()

    def same(got):
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(s["kc"], after[0]) and torch.equal(s["vc"], after[1])

    stream = torch.cuda.Stream()
    for given in (stream, stream.cuda_stream):
        reset()
        same(draft_step(s, given))
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = draft_step(s)
    for _ in range(3):
        reset()
        graph.replay()
        same(held)
        reset()
        same(draft_step(s))


def test_two_graphs_and_a_given_workspace():
    """Two captured calls with workspaces of their own, replayed in turn, and one workspace for calls one after another."""
    a, b = step_tensors("bf16", 0), step_tensors("bf16", 50)
    lib = __import__("paper_2609_38095_amd.decode", fromlist=["decode"])._lib()
    size = lib.zo_tree_attend_work(a["n"], 4, 8, 2, 64, zo.ZO_BF16)
    work = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    call = lambda s, **kw: zo.zo_tree_attend(s["q"], s["kc"], s["vc"], s["table"], s["lengths"], s["starts"], **kw)  # noqa: E731
    wants = [call(s, work=work) for s in (a, b)]
    assert torch.equal(wants[0], call(a)) and torch.equal(wants[1], call(b))
    graphs, held = [], []
    for s in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(call(s))
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], wants[0]) and torch.equal(held[1], wants[1])
        held[0].zero_(), held[1].zero_()


@pytest.mark.parametrize("dtype,dim,counts", [("bf16", 128, [300]), ("bf16", 64, [40]), ("bf16", 64, [600]), ("bf16", 256, [3, 2]), ("bf16", 256, [90]), ("f32", 128, [3, 2]), ("f32", 128, [90]),
                                              ("f32", 256, [50, 20]), ("f32", 64, [90]), ("f32", 64, [3]), ("bf16", 128, [3]), ("bf16", 64, [3]),
                                              ("f32", 96, [9])])
def test_every_form_in_graphs_and_at_once(dtype, dim, counts):
    """Each form of the kernel, first called inside a capture: its replays, and calls on two streams at once."""
    q, kc, vc, table, _ = attend_case([70] * len(counts), counts, 4, 2, dim, 16, "heads", dtype, 700)
    args = (kc, vc, dev(table), ints([70] * len(counts)), dev(starts_of(counts)))
    qs = [q, q.flip(0).contiguous()]
    graphs, held = [], []
    for x in qs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(zo.zo_tree_attend(x, *args))
    wants = [zo.zo_tree_attend(x, *args) for x in qs]
    for _ in range(3):
        for g, h in zip(graphs, held):
            h.zero_()
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(h, w) for h, w in zip(held, wants))
    streams, got = [torch.cuda.Stream() for _ in qs], []
    for _ in range(5):
        for x, stream in zip(qs, streams):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                got.append(zo.zo_tree_attend(x, *args))
    torch.cuda.synchronize()
    assert all(torch.equal(g, wants[i % 2]) for i, g in enumerate(got))


def test_drafted_trees_give_the_answers_of_single_tokens():
    """Trees of drafts, walked, kept and attended again: each walked token's result is that of a cache filled token by token."""
    torch.manual_seed(0)
    heads, dim, page, nodes = 2, 64, 4, 10
    book = zo.ZoPages(64, page)
    seq = book.add(5)
    kc, vc = cache_of("heads", 1, 64, heads, page, dim, "f32")
    turns = zo.zo_rotary_turns(dim)
    rng = np.random.default_rng(3)
    line_k, line_v = [kc[int(book.table([seq])[0][0, j // page]), :, j % page].clone() for j in range(5)], \
        [vc[int(book.table([seq])[0][0, j // page]), :, j % page].clone() for j in range(5)]
    for step in range(6):
        cached = book.length(seq)
        assert book.extend(seq, nodes) is None
        ids, _ = book.table([seq])
        parents = trees([nodes], step, 0.0)
        x = normal(step + 10, (nodes, 3 * heads, dim), "f32")
        q, k, v = x[:, :heads], x[:, heads:2 * heads], x[:, 2 * heads:]
        starts, lengths = ints([0, nodes]), ints([cached])
        seq_of, positions, places, seen = zo.zo_tree_lay(starts, lengths, nodes, dev(parents))
        qo, ko = zo.zo_norm_rotate(q, k, positions, turns)
        got = zo.zo_norm_rotate_put(q, k, v, kc, vc, dev(ids), positions, turns, seqs=seq_of, places=places)
        assert torch.equal(got, qo)
        out = zo.zo_tree_attend(got, kc, vc, dev(ids), lengths, starts, seen)
        drafted = rng.integers(0, 2, nodes).astype(np.int32)
        drawn = rng.integers(0, 2, nodes).astype(np.int32)
        path, _, counts = zo.zo_tree_accept(dev(drafted), dev(drawn), starts, nodes, dev(parents))
        zo.zo_tree_keep([kc], [vc], dev(ids), lengths, path)
        book.cut(seq, cached + int(counts[0]))
        for i in path[0, :int(counts[0])].tolist():
            line_k.append(ko[i]), line_v.append(v[i].clone())
            kk, vv = torch.stack(line_k).double(), torch.stack(line_v).double()
            w = torch.softmax(torch.einsum("thd,hd->ht", kk, qo[i].double()) * dim ** -0.5, -1)
            want = torch.einsum("ht,thd->hd", w, vv)
            assert float((out[i].double() - want).abs().max()) < 1e-5
    ids, lengths = book.table([seq])
    assert lengths[0] == len(line_k) and book.left() == 64 - -(-len(line_k) // page)
    for j in range(len(line_k)):
        assert torch.equal(kc[int(ids[0, j // page]), :, j % page], line_k[j])
        assert torch.equal(vc[int(ids[0, j // page]), :, j % page], line_v[j])


# ---- refusals

def test_refusals():
    s = step_tensors("bf16")
    q, kc, vc, table, lengths, starts = (s[n] for n in ("q", "kc", "vc", "table", "lengths", "starts"))
    n, out = s["n"], torch.full((s["n"], 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")

    def rejects(error, call, *args, **kw):
        with pytest.raises(error):
            call(*args, **kw)

    lay, attend, accept, keep = zo.zo_tree_lay, zo.zo_tree_attend, zo.zo_tree_accept, zo.zo_tree_keep
    rejects(TypeError, lay, starts.long(), lengths, n)
    rejects(TypeError, lay, starts, lengths, n, s["parents"].long())
    rejects(TypeError, lay, starts.cpu(), lengths, n)
    rejects(ValueError, lay, starts, lengths[:2], n)
    rejects(ValueError, lay, starts, lengths, n + 1, s["parents"])
    rejects(zo.ZoError, lay, starts, lengths, n, s["parents"], 0)
    rejects(zo.ZoError, lay, starts, lengths, n, s["parents"], 9)
    rejects(zo.ZoError, lay, starts, lengths, -1)
    rejects(zo.ZoError, lay, starts, lengths, 1 << 24)
    rejects(ValueError, lay, starts[:0], lengths, n)
    seen = torch.zeros(n, 1, dtype=torch.int64, device="cuda")
    rejects(TypeError, attend, q, kc, vc, table, lengths, starts, seen.int(), out=out)
    rejects(ValueError, attend, q, kc, vc, table, lengths, starts, seen[1:], out=out)
    rejects(ValueError, attend, q, kc, vc, table, lengths[1:], starts, out=out)
    rejects(ValueError, attend, q, kc, vc, table, lengths, starts[1:], out=out)
    rejects(ValueError, attend, q, kc, vc, table[1:], lengths, starts, out=out)
    rejects(ValueError, attend, q[..., :32], kc, vc, table, lengths, starts)
    rejects(TypeError, attend, q.float(), kc, vc, table, lengths, starts)
    rejects(TypeError, attend, q.half(), kc, vc, table, lengths, starts)
    rejects(zo.ZoError, attend, q[:, :7], kc, vc, table, lengths, starts)  # no multiple of the key heads
    rejects(zo.ZoError, attend, q, kc, vc, table, lengths, starts, scale=float("nan"), out=out)
    rejects(zo.ZoError, attend, q, kc, vc, table, lengths, starts, work=torch.empty(64, dtype=torch.uint8, device="cuda"), out=out)
    rejects(zo.ZoError, attend, q, kc, vc, table, lengths, starts, out=q)
    inside = kc.flatten()[:n * 64].view(n, 1, 64).expand(n, 8, 64)
    rejects(zo.ZoError, attend, q, kc, vc, table, lengths, starts, out=inside)
    assert bool((out == 7.0).all())
    rejects(zo.ZoError, accept, s["drafted"], s["drafted"], starts, 0)
    rejects(zo.ZoError, accept, s["drafted"], s["drafted"], starts, 1 << 23)
    rejects(ValueError, accept, s["drafted"], s["drafted"][1:], starts, 3)
    rejects(TypeError, accept, s["drafted"].long(), s["drafted"], starts, 3)
    path = torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    rejects(ValueError, keep, [kc], [vc], table, lengths, path[1:])
    rejects(ValueError, keep, [kc], [], table, lengths, path)
    rejects(TypeError, keep, [kc], [vc], table, lengths, path.long())
    buffer = torch.zeros(17, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    rejects(zo.ZoError, keep, [buffer[:16]], [buffer[1:]], table, lengths, path)  # caches that overlap
    keep([], [], table, lengths, path)


def test_nothing_to_do():
    s = step_tensors("f32")
    none = ints([])
    assert [t.numel() for t in zo.zo_tree_lay(ints([0]), none, 0)[:3]] == [0, 0, 0]
    assert zo.zo_tree_attend(s["q"][:0], s["kc"], s["vc"], s["table"], s["lengths"], ints([0] * 5)).shape == (0, 8, 64)
    path, tokens, counts = zo.zo_tree_accept(none, none, ints([0, 0, 0]), 3)
    assert path.tolist() == [[-1] * 3] * 2 and tokens.tolist() == [[-1] * 3] * 2 and counts.tolist() == [0, 0]
    before = s["kc"].clone()
    zo.zo_tree_keep([s["kc"]], [s["vc"]], s["table"], s["lengths"], torch.empty(4, 0, dtype=torch.int32, device="cuda"))
    assert torch.equal(s["kc"], before)
    # masks without words: the cached tokens alone
    got = zo.zo_tree_attend(s["q"], s["kc"], s["vc"], s["table"], s["lengths"], s["starts"], torch.empty(s["n"], 0, dtype=torch.int64, device="cuda"))
    zero = torch.zeros(s["n"], 1, dtype=torch.int64, device="cuda")
    assert torch.equal(got, zo.zo_tree_attend(s["q"], s["kc"], s["vc"], s["table"], s["lengths"], s["starts"], zero))
