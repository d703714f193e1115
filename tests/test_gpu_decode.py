"""The decode-step operators on the GPU against the oracle in 64 bits.

Tolerances follow from the arithmetic, with e = 2^-24 (half an fp32 ulp, relative). Rows: a norm's sum
of squares, root, two products and a turned pair are below 32 e of the magnitudes that feed an
element (angles are exact to 2 pi 2^-26, 2 e); gradients add a sum of dim products, below 64 e; a
gamma's gradient is a sum over rows of which no partial sum is longer than a few dozen, below 128 e.
Attention: a score is a sum of dim products, off by at most (dim + 8) e of its products' magnitudes, which
moves each weight by that share, twice (weight and sum); running sums add a rounding for each tile. A
bf16 result adds half a bf16 ulp, bf16 weights two parts of 8 bits each (2^-16 of the weight, 2^8 e).
"""

import math

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
from oracle import decode as oracle

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def wide(t):
    return t.detach().double().cpu().numpy()


def near(got, want, magnitude, steps, dtype):
    got = wide(got)
    assert np.array_equal(np.isfinite(got), np.isfinite(want))
    off = np.abs(got - want)
    # half a bf16 ulp: 8 significant bits, so 2^-8 of the power of two at or below the value
    half_ulp = np.exp2(np.floor(np.log2(np.maximum(np.abs(np.where(np.isfinite(want), want, 1.0)), 1e-38))) - 8)
    most = steps * E * magnitude + (half_ulp if dtype == "bf16" else 0.0) + 1e-37
    worst = np.nanmax(np.where(np.isfinite(want), off / most, 0.0)) if off.size else 0.0
    assert worst <= 1.0, f"off by {worst:.2f} of what rounding allows"


def normal(seed, shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0, scale, generator=g).to(TYPES[dtype])


def rows_of(kind, seed, tokens, hq, hk, dim, dtype):
    """q, k, v as tensors of their own, views of one projection, head-major views, or views that begin one
    element behind a vector's boundary."""
    if kind == "own":
        return [normal(seed + i, (tokens, h, dim), dtype) for i, h in enumerate((hq, hk, hk))]
    if kind == "fused":
        x = normal(seed, (tokens, hq + 2 * hk, dim), dtype)
        return [x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]]
    if kind == "heads":
        return [normal(seed + i, (h, tokens, dim), dtype).transpose(0, 1) for i, h in enumerate((hq, hk, hk))]
    x = normal(seed, (tokens, hq + 2 * hk, dim + 3), dtype)[:, :, 1:1 + dim]
    return [x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]]


ROWS = [
    # tokens, q heads, k heads, dim, rotated, interleaved, norm, views, positions up to
    (1, 1, 1, 2, 2, False, True, "own", 10),
    (3, 5, 3, 1, 0, False, True, "own", 10),
    (7, 4, 2, 6, 4, False, True, "own", 1000),
    (7, 4, 2, 6, 4, True, True, "fused", 1000),
    (33, 5, 3, 16, 16, True, True, "own", 100),
    (33, 3, 1, 48, 32, False, True, "heads", 100),
    (19, 12, 12, 64, 64, False, False, "fused", 2050),
    (19, 12, 4, 64, 32, True, True, "odd", 2050),
    (65, 2, 1, 80, 80, False, True, "odd", 5000),
    (65, 2, 1, 80, 40, True, True, "fused", 5000),
    (50, 6, 2, 96, 96, False, True, "fused", 5000),
    (50, 6, 2, 100, 50, False, True, "own", 5000),
    (129, 32, 8, 128, 128, False, True, "fused", 40000),
    (129, 16, 8, 128, 128, True, True, "heads", 2 ** 31 - 200),
    (700, 40, 1, 128, 64, False, True, "own", 300000),
    (2048, 1, 1, 128, 128, False, True, "own", 4096),
    (257, 3, 2, 256, 256, False, True, "fused", 100),
    (257, 3, 2, 255, 254, True, True, "own", 100),
    (4099, 8, 4, 64, 64, False, True, "fused", 4099),
    (8192, 8, 4, 128, 128, False, True, "fused", 8192),  # several rows for each lane group from here on
    (20_001, 4, 4, 64, 32, True, True, "own", 30_000),
    (2101, 2, 2, 50, 50, False, True, "odd", 3000),
    (3001, 4, 2, 256, 128, False, True, "heads", 3000),
    (5, 4, 0, 64, 64, False, True, "own", 5),
    (5, 0, 4, 64, 0, False, True, "own", 5),
]


def rotate_case(case, dtype):
    tokens, hq, hk, dim, rotary, interleaved, norm, views, far = case
    q, k, v = rows_of(views, 11, tokens, hq, hk, dim, dtype)
    rng = np.random.default_rng(tokens)
    at = rng.integers(0, far, tokens).astype(np.int32)
    at[-1] = far - 1
    if tokens > 2:
        at[1] = -1  # padding, whatever it holds
        for t in (q, k):
            t[1] = float("nan")
    turns = zo.zo_rotary_turns(rotary, 1e4) if rotary else None
    gq = 1 + normal(5, (dim,), dtype, 0.1) if norm else None
    gk = 1 + normal(6, (dim,), dtype, 0.1) if norm and hk != 2 else None  # one side may go without
    kw = dict(turns=turns, interleaved=interleaved, magnitude=0.7 if views == "own" else 1.0)
    return q, k, v, torch.from_numpy(at).cuda(), at, gq, gk, kw


def exact_rows(x, gamma, at, kw, eps=1e-6):
    return oracle.norm_rotate(wide(x), None if gamma is None else wide(gamma), at,
                              kw["turns"] if kw["turns"] is not None else np.zeros(0), kw["interleaved"], kw["magnitude"], eps)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", ROWS)
def test_norm_rotate(case, dtype):
    q, k, v, positions, at, gq, gk, kw = rotate_case(case, dtype)
    qo, ko = zo.zo_norm_rotate(q if case[1] else None, k if case[2] else None, positions, q_gamma=gq, k_gamma=gk, **kw)
    wants = []
    for got, x, g in ((qo, q, gq), (ko, k, gk)):
        if x.shape[1] == 0:
            assert got is None
            continue
        want, magnitude = exact_rows(x, g, at, kw)
        near(got, want, magnitude, 32, dtype)
        wants.append(got)
    # in place, bit for bit the same
    if case[1] and case[2]:
        zo.zo_norm_rotate(q, k, positions, q_gamma=gq, k_gamma=gk, q_out=q, k_out=k, **kw)
        assert torch.equal(q, wants[0]) and torch.equal(k, wants[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", ROWS)
def test_norm_rotate_back(case, dtype):
    q, k, v, positions, at, gq, gk, kw = rotate_case(case, dtype)
    dqo, dko, _ = rows_of("own", 77, case[0], case[1], case[2], case[3], dtype)
    hq, hk = case[1], case[2]
    got = zo.zo_norm_rotate_back(dqo if hq else None, dko if hk else None, q if hq else None, k if hk else None, positions,
                                 q_gamma=gq, k_gamma=gk, **kw)
    again = zo.zo_norm_rotate_back(dqo if hq else None, dko if hk else None, q if hq else None, k if hk else None, positions,
                                   q_gamma=gq, k_gamma=gk, **kw)
    for one, two in zip(got, again):
        assert (one is None) == (two is None) and (one is None or torch.equal(one, two))
    for dx, dg, dy, x, g in ((got[0], got[2], dqo, q, gq), (got[1], got[3], dko, k, gk)):
        if x.shape[1] == 0:
            assert dx is None and dg is None
            continue
        turns = kw["turns"] if kw["turns"] is not None else np.zeros(0)
        want, mag, want_g, mag_g = oracle.norm_rotate_back(wide(dy), wide(x), None if g is None else wide(g), at, turns,
                                                           kw["interleaved"], kw["magnitude"])
        near(dx, want, mag, 64, dtype)
        if g is None:
            assert dg is None
        else:
            assert dg.dtype == torch.float32
            near(dg, want_g, mag_g, 128, "f32")


def test_norm_rotate_back_against_differences():
    """A directional derivative of the forward kernel: central differences of sum(w y) in a step of 2^-7
    are off by the cubic term and by rounding over the step, both far below 1e-3 of sum |w y|."""
    q, k, v, positions, at, gq, gk, kw = rotate_case((65, 4, 2, 128, 64, False, True, "own", 5000), "f32")
    q[1] = 0.0
    w, direction, dgamma = normal(1, q.shape, "f32"), normal(2, q.shape, "f32"), normal(3, gq.shape, "f32")
    h = 2.0 ** -7
    def loss(x, g):
        return float((zo.zo_norm_rotate(x, None, positions, q_gamma=g, **kw)[0].double() * w.double()).sum())
    dq, _, dg, _ = zo.zo_norm_rotate_back(w, None, q, None, positions, q_gamma=gq, **kw)
    size = float((zo.zo_norm_rotate(q, None, positions, q_gamma=gq, **kw)[0] * w).abs().sum())
    moved = (loss(q + h * direction, gq) - loss(q - h * direction, gq)) / (2 * h)
    assert abs(moved - float((dq.double() * direction.double()).sum())) <= 1e-3 * size
    moved = (loss(q, gq + h * dgamma) - loss(q, gq - h * dgamma)) / (2 * h)
    assert abs(moved - float((dg.double() * dgamma.double()).sum())) <= 1e-3 * size


def test_norm_rotate_back_without_tokens():
    x = torch.empty(0, 4, 64, device="cuda")
    g = torch.ones(64, device="cuda")
    dq, _, dg, _ = zo.zo_norm_rotate_back(x, None, x, None, torch.empty(0, dtype=torch.int32, device="cuda"), q_gamma=g)
    assert dq.shape == (0, 4, 64) and torch.equal(dg, torch.zeros_like(g))


def scattered(lengths, page, pages, width, rng, absent=()):
    table = np.full((len(lengths), width), -1, np.int32)
    ids = rng.permutation(pages)
    at = 0
    for s, n in enumerate(lengths):
        need = min(max(-(-int(n) // page), 0), width)
        table[s, :need] = ids[at:at + need]
        at += need
    for s, j, what in absent:
        table[s, j] = what
    return table


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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,rotary,page,layout", [(128, 128, 16, "heads"), (64, 32, 48, "tokens"), (6, 4, 3, "both"),
                                                    (96, 96, 1, "odd"), (256, 0, 64, "both")])
def test_norm_rotate_put(dim, rotary, page, layout, dtype):
    rng = np.random.default_rng(3)
    seqs, hq, hk, width = 5, 6, 3, 4
    # tokens of sequences in any order: prompts, single tokens, padding, places that there are not
    seq = np.array([0] * 7 + [1, 2, 2, 3, 4, 5, 77, 4, 4], np.int32)
    at = np.array(list(range(7)) + [2, 5, -1, width * page - 1, 0, 1, 1, width * page, 3], np.int32)
    n = len(seq)
    table = scattered([width * page] * seqs, page, seqs * width + 2, width, rng, [(2, min(5 // page, width - 1), -1), (4, 3 // page, seqs * width + 2)])
    kc, vc = cache_of(layout, 5, seqs * width + 2, hk, page, dim, dtype)
    before = [kc.clone(), vc.clone()]
    q, k, v = rows_of("fused", 9, n, hq, hk, dim, dtype)
    turns = zo.zo_rotary_turns(rotary, 1e4) if rotary else None
    gq, gk = (1 + normal(i, (dim,), dtype, 0.1) for i in (1, 2))
    positions, dev_seq = torch.from_numpy(at).cuda(), torch.from_numpy(seq).cuda()
    got = zo.zo_norm_rotate_put(q, k, v, kc, vc, torch.from_numpy(table).cuda(), positions, turns, q_gamma=gq, k_gamma=gk,
                                seqs=dev_seq)
    qo, ko = zo.zo_norm_rotate(q, k, positions, turns, q_gamma=gq, k_gamma=gk)
    assert torch.equal(got, qo)
    for t in range(n):
        if at[t] < 0 or seq[t] >= seqs or at[t] >= width * page:
            continue
        p = table[seq[t], at[t] // page]
        if 0 <= p < seqs * width + 2:
            before[0][p, :, at[t] % page] = ko[t]
            before[1][p, :, at[t] % page] = v[t]
    assert torch.equal(kc, before[0]) and torch.equal(vc, before[1])
    # without queries, token t into sequence t
    kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vc)
    assert zo.zo_norm_rotate_put(None, k[:seqs], v[:seqs], kc2, vc2, torch.from_numpy(table).cuda(), positions[:seqs], turns,
                                 k_gamma=gk) is None
    for t in range(seqs):
        if at[t] < width * page and 0 <= (p := table[t, at[t] // page]) < seqs * width + 2:
            assert torch.equal(kc2[p, :, at[t] % page], ko[t]) and torch.equal(vc2[p, :, at[t] % page], v[t])


ATTEND = [
    # lengths, width of the table, q heads, k heads, dim, page, layout, scale
    ([1], 1, 1, 1, 64, 16, "heads", None),
    ([0, 0], 2, 4, 2, 64, 16, "heads", None),
    ([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65], 5, 4, 4, 64, 16, "heads", None),
    ([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65], 5, 12, 3, 128, 16, "tokens", None),
    ([5, 3000, 1], 64, 8, 2, 128, 48, "both", 0.3),
    ([4500, 7], 48, 32, 8, 128, 96, "heads", None),
    ([700, 0, 33], 8, 17, 1, 64, 128, "tokens", None),
    ([257], 17, 40, 1, 128, 16, "heads", None),
    ([130, 2], 9, 3, 3, 256, 16, "both", None),
    ([300, 20], 20, 6, 2, 128, 16, "odd", None),
    ([70, 20, 3], 25, 4, 2, 1, 3, "heads", 1.0),
    ([70, 0, 33], 70, 4, 2, 20, 1, "both", None),
    ([70, 5, 33], 5, 6, 2, 80, 16, "odd", None),
    ([90, 5, 33], 4, 6, 2, 128, 24, "tokens", None),
    ([90, 5, 33], 4, 2, 1, 200, 24, "tokens", None),
    ([120, 64], 8, 4, 2, 128, 16, "heads", 0.0),
    ([120, 64], 8, 4, 2, 64, 16, "heads", -0.2),
    ([400, -3, 10 ** 9], 6, 4, 2, 128, 64, "heads", 2.0),
]


def attend_bound(dim, longest, big, dtype):
    """Steps of rounding behind an output, relative to the weighted magnitudes of the values."""
    return 2 * (dim + 8) * big + longest / 16 + 64 + (2.0 ** 8 if dtype == "bf16" else 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", ATTEND, ids=[str(i) for i in range(len(ATTEND))])
def test_cache_attend(case, dtype):
    lengths, width, hq, hk, dim, page, layout, scale = case
    rng = np.random.default_rng(len(lengths))
    pages = len(lengths) * width + 3
    table = scattered(lengths, page, pages, width, rng)
    kc, vc = cache_of(layout, 21, pages, hk, page, dim, dtype)
    q = normal(3, (len(lengths), hq, dim), dtype, 1.5)
    scale = dim ** -0.5 if scale is None else scale
    want, lse, mag, big = oracle.attend(wide(q), wide(kc), wide(vc), table, lengths, scale)
    # whatever lies behind the ends, in pages of no one or in absent ones, is not read
    for s, n in enumerate(lengths):
        n = min(max(n, 0), width * page)
        if n % page:
            kc[table[s, n // page], :, n % page:] = float("nan")
            vc[table[s, n // page], :, n % page:] = float("inf")
    for p in set(range(pages)) - set(table.reshape(-1).tolist()):
        kc[p], vc[p] = float("nan"), float("nan")
    dev = torch.from_numpy(table).cuda(), torch.from_numpy(np.array(lengths, np.int32)).cuda()
    out, sums = zo.zo_cache_attend(q, kc, vc, *dev, scale, lse=True)
    steps = attend_bound(dim, 4500, big, dtype)
    near(out, want, mag, steps[..., None], dtype)
    assert np.array_equal(np.isneginf(wide(sums)), np.isneginf(lse))
    fine = np.isfinite(lse)
    assert np.all(np.abs(wide(sums)[fine] - lse[fine]) <= (steps[fine] + 8 * np.abs(lse[fine])) * E)
    assert torch.equal(out, zo.zo_cache_attend(q, kc, vc, *dev, scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,dim", [(16, 64), (32, 128), (5, 64)])
def test_cache_attend_absent_pages(page, dim, dtype):
    """Ids outside the cache leave their tokens out; a sequence of nothing else is empty."""
    rng = np.random.default_rng(8)
    lengths, width, pages = [10 * page, 3 * page + 2, 2 * page, page - 1], 10, 40
    table = scattered(lengths, page, pages, width, rng,
                      [(0, 0, -1), (0, 3, pages), (0, 4, 2 ** 31 - 1), (0, 9, -2 ** 31), (1, 3, -7), (2, 0, -1), (2, 1, -1)])
    kc, vc = cache_of("heads", 2, pages, 2, page, dim, dtype)
    q = normal(3, (4, 4, dim), dtype)
    want, lse, mag, big = oracle.attend(wide(q), wide(kc), wide(vc), table, lengths, 0.2)
    used = {int(p) for p in table.reshape(-1) if 0 <= p < pages}
    for p in set(range(pages)) - used:
        kc[p], vc[p] = float("inf"), float("nan")
    out, sums = zo.zo_cache_attend(q, kc, vc, torch.from_numpy(table).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), 0.2,
                                   lse=True)
    near(out, want, mag, attend_bound(dim, 160, big, dtype)[..., None], dtype)
    assert torch.equal(out[2], torch.zeros_like(out[2])) and bool(torch.isneginf(sums[2]).all())


@pytest.mark.parametrize("seqs", [255, 257, 1000])
def test_cache_attend_many_sequences(seqs):
    """More sequences than a workgroup has threads; some empty, one long."""
    rng = np.random.default_rng(seqs)
    lengths = rng.integers(0, 40, seqs)
    lengths[rng.random(seqs) < 0.3] = 0
    lengths[seqs // 2] = 2000
    width, page = 125, 16
    pages = int((-(-lengths // page)).sum()) + 1
    table = scattered(lengths, page, pages, width, rng)
    kc, vc = cache_of("heads", 4, pages, 2, page, 64, "bf16")
    q = normal(5, (seqs, 4, 64), "bf16")
    want, lse, mag, big = oracle.attend(wide(q), wide(kc), wide(vc), table, lengths, 0.125)
    out = zo.zo_cache_attend(q, kc, vc, torch.from_numpy(table).cuda(), torch.from_numpy(lengths.astype(np.int32)).cuda())
    near(out, want, mag, attend_bound(64, 2000, big, "bf16")[..., None], "bf16")


def test_cache_attend_far_pages():
    """Offsets that pass 2^31 elements: a cache of 2.3 G elements, keys and values the same."""
    pages, heads, page, dim = 70_000, 16, 16, 128
    c = torch.empty(pages, heads, page, dim, dtype=torch.bfloat16, device="cuda")
    ids = [69_999, 66_000, 12, 65_536]
    for i in ids:
        c[i] = normal(i, (heads, page, dim), "bf16")
    q = normal(1, (1, 32, dim), "bf16")
    table = torch.tensor([ids], dtype=torch.int32)
    few = c[ids].clone()
    out = zo.zo_cache_attend(q, c, c, table.cuda(), torch.tensor([60], dtype=torch.int32).cuda())
    want, _, mag, big = oracle.attend(wide(q), wide(few), wide(few), np.array([[0, 1, 2, 3]]), [60], dim ** -0.5)
    near(out, want, mag, attend_bound(dim, 60, big, "bf16")[..., None], "bf16")
    k, v = normal(7, (1, heads, dim), "bf16"), normal(8, (1, heads, dim), "bf16")
    zo.zo_norm_rotate_put(None, k, v, c, c.clone(), table.cuda(), torch.tensor([20], dtype=torch.int32).cuda())
    assert torch.equal(c[66_000, :, 4], k[0]) and torch.equal(c[66_000, :, 3], few[1, :, 3])


def test_cache_attend_infinite_values():
    """An infinite value reaches its own sequence's output and no other's; so does a NaN."""
    kc, vc = cache_of("heads", 2, 8, 1, 16, 64, "bf16")
    q = normal(3, (2, 2, 64), "bf16")
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([20, 20], dtype=torch.int32, device="cuda")
    plain = zo.zo_cache_attend(q, kc, vc, table, lengths)
    vc[0, 0, 3, 5] = float("inf")
    vc[1, 0, 2, 9] = float("nan")
    out = zo.zo_cache_attend(q, kc, vc, table, lengths)
    assert torch.equal(out[1], plain[1])
    assert bool((out[0, :, 5] == float("inf")).all()) and bool(out[0, :, 9].isnan().all())
    rest = [i for i in range(64) if i not in (5, 9)]
    assert torch.equal(out[0][:, rest], plain[0][:, rest])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,dim,page,layout", [(8, 128, 16, "heads"), (12, 64, 48, "tokens"), (3, 20, 5, "both"), (2, 17, 7, "odd")])
def test_cache_copy(heads, dim, page, layout, dtype):
    rng = np.random.default_rng(4)
    layers, pages, n = 3, 700, 250  # more moves than a launch holds
    caches = [cache_of(layout, 10 * i, pages, heads, page, dim, dtype) for i in range(layers)]
    want = [[t.clone() for t in c] for c in caches]
    order = rng.permutation(pages)
    src, dst = order[:n], order[n:2 * n]
    src[5] = src[6]  # one page to two
    rows = rng.integers(1, page + 1, n)
    for c in want:
        for t in c:
            for a, b, r in zip(src.tolist(), dst.tolist(), rows.tolist()):
                t[b, :, :r] = t[a, :, :r]
    zo.zo_cache_copy([c[0] for c in caches], [c[1] for c in caches], src, dst, rows)
    for c, w in zip(caches, want):
        assert torch.equal(c[0], w[0]) and torch.equal(c[1], w[1])


def test_cache_copy_many_layers():
    """More layers than a launch holds; whole pages."""
    caches = [cache_of("heads", i, 6, 1, 16, 8, "f32") for i in range(70)]
    want = [[t[2].clone() for t in c] for c in caches]
    zo.zo_cache_copy([c[0] for c in caches], [c[1] for c in caches], [2, 2], [4, 0])
    for c, w in zip(caches, want):
        for t, p in zip(c, w):
            assert torch.equal(t[4], p) and torch.equal(t[0], p)


def test_pages_fork_compact_and_attend():
    """Forked, grown and compacted sequences attend to what they hold."""
    page, heads, dim, layers = 4, 2, 64, 2
    book = zo.ZoPages(64, page)
    caches = [cache_of("heads", 3 * i, 64, heads, page, dim, "f32") for i in range(layers)]
    held = {}  # sequence -> its keys and values, token by token
    rng = np.random.default_rng(0)

    def grow(seq, n):
        for _ in range(n):
            move = book.extend(seq)
            if move:
                zo.zo_cache_copy([c[0] for c in caches], [c[1] for c in caches], [move[0]], [move[1]], [move[2]])
            ids, lengths = book.table([seq])
            k, v = (torch.from_numpy(rng.standard_normal((1, heads, dim)).astype(np.float32)).cuda() for _ in range(2))
            for kc, vc in caches:
                zo.zo_norm_rotate_put(None, k, v, kc, vc, torch.from_numpy(ids).cuda(), torch.from_numpy(lengths - 1).cuda())
            held[seq].append((k, v))

    def check():
        seqs = sorted(held)
        ids, lengths = book.table(seqs)
        assert lengths.tolist() == [len(held[s]) for s in seqs]
        for kc, vc in caches:
            for s, row in zip(seqs, ids):
                for j, (k, v) in enumerate(held[s]):
                    assert torch.equal(kc[row[j // page], :, j % page], k[0]) and torch.equal(vc[row[j // page], :, j % page], v[0])

    a = book.add()
    held[a] = []
    grow(a, 10)
    b, c = book.fork(a), book.fork(a)
    held[b], held[c] = list(held[a]), list(held[a])
    grow(b, 3)
    grow(a, 1)
    grow(c, 7)
    check()
    book.drop(a)
    del held[a]
    d = book.fork(c)
    held[d] = list(held[c])
    src, dst, rows = book.compact()
    assert len(src) > 0
    zo.zo_cache_copy([x[0] for x in caches], [x[1] for x in caches], src, dst, rows)
    ids, _ = book.table(sorted(held))
    assert ids.max() < 64 - book.left()
    check()
    grow(d, 5)
    grow(c, 5)
    check()


def draw_rows(kind, rows, vocab, dtype, seed=0):
    x = normal(seed, (rows, vocab), "f32", 2.0)
    if kind == "peaked":
        x[:, ::max(1, vocab // 40)] += 8.0
    elif kind == "ties":
        x = torch.round(x)
    elif kind == "flat":
        x = torch.zeros_like(x)
        x[:, ::2] = -0.0  # equal to 0
    elif kind == "masked":
        x[:, vocab // 3:] = -math.inf
        x[0] = -math.inf
        x[1 % rows] = float("nan")
        x[2 % rows, ::3] = float("nan")
        x[3 % rows, vocab - 1] = math.inf
        x[3 % rows, vocab // 2] = math.inf
        x[4 % rows] = torch.finfo(TYPES[dtype]).min
    elif kind == "steep":
        x = x * 1e4
    return x.to(TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,vocab", [("peaked", 1), ("peaked", 2), ("ties", 7), ("peaked", 511), ("flat", 512), ("masked", 513),
                                        ("ties", 1009), ("peaked", 1009), ("steep", 1009), ("flat", 5000), ("masked", 5000),
                                        ("ties", 50_272), ("peaked", 50_272), ("flat", 50_272), ("peaked", 151_936), ("peaked", 1 << 18)])
def test_draw(kind, vocab, dtype):
    settings = [  # temperature, top_k, top_p, min_p, u
        (1.0, 0, 1.0, 0.0, 0.5), (0.7, 0, 1.0, 0.0, 0.0), (1.3, 0, 1.0, 0.0, 0.99999994), (1.0, 1, 1.0, 0.0, 0.7),
        (1.0, 3, 1.0, 0.0, 0.9), (0.8, 40, 0.9, 0.0, 0.3), (1.0, 0, 0.95, 0.0, 0.6), (2.0, 0, 0.5, 0.0, 0.8),
        (1.0, 0, 0.0, 0.0, 0.8), (1.0, 0, 1.0, 0.05, 0.8), (1.0, 0, 1.0, 1.0, 0.8), (1.0, 50, 0.99, 0.3, 1.0),
        (0.0, 5, 0.5, 0.0, 0.5), (-1.0, 0, 1.0, 0.0, 0.5), (float("nan"), 0, 1.0, 0.0, 0.5), (1.0, vocab + 5, 1.5, -1.0, -3.0),
        (1.0, 700, 0.999, 0.0, 0.123), (3.0, 2000, 0.97, 7.0, 0.999), (1e-30, 0, 0.9, 0.0, 0.5), (1e30, 0, 0.9, 0.0, 0.5),
        (1.0, -2, 0.3, 0.0, float("nan")),
    ]
    if vocab > 10_000:
        settings = settings[:9] + settings[11:13] + settings[16:17]
    rows = len(settings)
    x = draw_rows(kind, rows, vocab, dtype)
    wide_row = torch.zeros(rows, vocab + 3, dtype=x.dtype, device="cuda")
    wide_row[:, 1:1 + vocab] = x
    x = wide_row[:, 1:1 + vocab]  # rows apart, begun off a vector's boundary
    t, k, p, m, u = (torch.tensor(c, dtype=torch.int32 if i == 1 else torch.float32, device="cuda") for i, c in enumerate(zip(*settings)))
    token, logprob = zo.zo_draw(x, u, t, k, p, m, logprobs=True)
    host = x.float().cpu().numpy()
    for b, (ti, ki, pi, mi, ui) in enumerate(settings):
        want, lp = oracle.draw(host[b], ui, ti, ki, pi, mi)
        assert int(token[b]) == want, (b, settings[b])
        got = float(logprob[b])
        assert got == lp or abs(got - lp) <= 4 * E * max(1.0, abs(lp)), (b, settings[b])


def test_draw_without_settings_follows_the_distribution():
    """100,000 draws of one row of 5 logits: each share within 5 standard deviations."""
    n = 100_000
    x = torch.tensor([[0.3, -1.0, 1.7, 0.0, -2.0]], device="cuda").expand(n, 5)  # one row, broadcast
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    token = zo.zo_draw(x, torch.rand(n, generator=g, device="cuda"))
    want = torch.softmax(x[0].double(), 0).cpu().numpy()
    got = np.bincount(token.cpu().numpy(), minlength=5) / n
    assert np.all(np.abs(got - want) <= 5 * np.sqrt(want * (1 - want) / n))


def test_streams_and_graphs():
    """A whole decode step on a stream of its own, and captured: replays give the eager step's bits, with other
    work between them."""
    seqs, hq, hk, dim, page, vocab = 6, 8, 2, 64, 16, 1009
    width = 4
    q, k, v = rows_of("fused", 3, seqs, hq, hk, dim, "bf16")
    kc, vc = cache_of("heads", 1, seqs * width, hk, page, dim, "bf16")
    table = torch.arange(seqs * width, dtype=torch.int32, device="cuda").reshape(seqs, width)
    positions = torch.tensor([0, 5, 15, 16, 40, 63], dtype=torch.int32, device="cuda")
    lengths = positions + 1
    logits, u = normal(9, (seqs, vocab), "bf16", 3.0), torch.linspace(0, 0.99, seqs, device="cuda")
    gamma = torch.ones(dim, dtype=torch.bfloat16, device="cuda")
    k_args = torch.full((seqs,), 20, dtype=torch.int32, device="cuda")
    turns = zo.zo_rotary_turns(dim, 1e6)
    first = kc.clone(), vc.clone()

    def step(stream=None):
        qo = zo.zo_norm_rotate_put(q, k, v, kc, vc, table, positions, turns, q_gamma=gamma, k_gamma=gamma, stream=stream)
        out = zo.zo_cache_attend(qo, kc, vc, table, lengths, stream=stream)
        zo.zo_cache_copy([kc], [vc], [0], [1], stream=stream)
        return qo, out, zo.zo_draw(logits, u, top_k=k_args, stream=stream), kc.clone(), vc.clone()

    want = step()
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(),):
        for given in (stream, stream.cuda_stream):
            kc.copy_(first[0]), vc.copy_(first[1])
            torch.cuda.synchronize()
            got = step(given)[:3]
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b)
            assert torch.equal(kc, want[3]) and torch.equal(vc, want[4])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        kc.copy_(first[0]), vc.copy_(first[1])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)
        assert torch.equal(step()[1], want[1])


def test_refusals():
    """Wrong arguments raise and leave the outputs as they were."""
    q, k, v = rows_of("own", 1, 4, 6, 2, 64, "bf16")
    kc, vc = cache_of("heads", 2, 8, 2, 16, 64, "bf16")
    at = torch.arange(4, dtype=torch.int32, device="cuda")
    table = torch.arange(8, dtype=torch.int32, device="cuda").reshape(4, 2)
    lengths = at + 1
    out = torch.full_like(q, 7.0)
    turns = zo.zo_rotary_turns(64)

    def rejects(error, call, *args, **kw):
        with pytest.raises(error):
            call(*args, **kw)

    rotate = zo.zo_norm_rotate
    rejects(TypeError, rotate, q, k.float(), at)
    rejects(TypeError, rotate, q, k, at.long())
    rejects(TypeError, rotate, q, k, at, turns.astype(np.float32).reshape(2, -1))
    rejects(TypeError, rotate, q, k.cpu(), at)
    rejects(TypeError, rotate, q, k, at, q_gamma=torch.ones(64, device="cuda"))
    rejects(ValueError, rotate, q, k[:, :, :32], at)
    rejects(ValueError, rotate, q, k[:3], at)
    rejects(ValueError, rotate, q, k, at[:3])
    rejects(ValueError, rotate, q.transpose(1, 2), None, at)
    rejects(ValueError, rotate, q, k, at, q_out=out[:3])
    rejects(ValueError, rotate, None, None, at)
    for bad, code in ((dict(turns=zo.zo_rotary_turns(66)), zo.ZO_ERR_ARG), (dict(norm_eps=float("nan")), zo.ZO_ERR_NONFINITE),
                      (dict(q_out=out.expand(4, 6, 64)[:1].expand(4, 6, 64)), zo.ZO_ERR_ARG),  # rows that overlap
                      (dict(q_out=q[:, :, :].flip(1).flip(1).as_strided((4, 6, 64), (384, 64, 1)), turns=turns * np.inf), zo.ZO_ERR_NONFINITE)):
        with pytest.raises(zo.ZoError) as e:
            rotate(q, k, at, **bad)
        assert e.value.status == code
    shifted = torch.zeros(4 * 6 * 64 + 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(zo.ZoError):  # an output that begins an element behind its input
        rotate(shifted[:-1].view(4, 6, 64), None, at, q_out=shifted[1:].view(4, 6, 64))
    attend = zo.zo_cache_attend
    rejects(TypeError, attend, q.float(), kc, vc, table, lengths)
    rejects(TypeError, attend, q, kc, vc, table.long(), lengths)
    rejects(ValueError, attend, q, kc, vc[:4], table, lengths)
    rejects(ValueError, attend, q, kc, vc, table[:2], lengths)
    rejects(ValueError, attend, q, kc, vc, table, lengths[:2])
    rejects(ValueError, attend, q[:, :, :32], kc, vc, table, lengths)
    rejects(zo.ZoError, attend, q[:, :3], kc, vc, table, lengths)  # 3 query heads for 2 key heads
    rejects(zo.ZoError, attend, q, kc, vc, table, lengths, float("inf"), out=out)
    rejects(zo.ZoError, attend, q, kc, vc, table, lengths, out=out, work=torch.empty(64, dtype=torch.uint8, device="cuda"))
    rejects(zo.ZoError, attend, q, kc, vc, table, lengths, out=q)
    rejects(ValueError, zo.zo_norm_rotate_put, q, k, v, kc, vc.transpose(0, 1), table, at)
    rejects(zo.ZoError, zo.zo_norm_rotate_put, q, k[:, :1], v[:, :1], kc, vc, table, at)  # another count of heads
    back = zo.zo_norm_rotate_back
    gamma = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    rejects(TypeError, back, out, None, None, None, at, q_gamma=gamma)  # the input is needed with a gamma
    rejects(zo.ZoError, back, out, None, q, None, at, q_gamma=gamma, work=torch.empty(16, dtype=torch.uint8, device="cuda"))
    rejects(zo.ZoError, zo.zo_cache_copy, [kc], [vc], [0, 1], [1, 2])
    rejects(zo.ZoError, zo.zo_cache_copy, [kc], [vc], [0], [8])
    rejects(ValueError, zo.zo_cache_copy, [kc], [vc], [0, 1], [2])
    rejects(ValueError, zo.zo_cache_copy, [kc, kc[:4]], [vc, vc[:4]], [0], [1])
    logits, u = normal(1, (4, 100), "f32"), torch.rand(4, device="cuda")
    rejects(TypeError, zo.zo_draw, logits, u.double())
    rejects(TypeError, zo.zo_draw, logits, u, top_k=torch.ones(4, device="cuda"))
    rejects(ValueError, zo.zo_draw, logits, u[:3])
    rejects(ValueError, zo.zo_draw, logits.T, u)
    rejects(zo.ZoError, zo.zo_draw, logits[:, :0], u)
    if torch.cuda.device_count() == 1:
        stream = torch.cuda.Stream()
        rejects(TypeError, zo.zo_draw, logits.cpu(), u, stream=stream)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


def test_work_and_outputs_given():
    """Results in given tensors, with given workspaces, are those of the allocated ones."""
    q, k, _ = rows_of("fused", 5, 9, 4, 2, 64, "f32")
    kc, vc = cache_of("tokens", 6, 40, 2, 16, 64, "f32")
    table = torch.arange(36, dtype=torch.int32, device="cuda").reshape(9, 4)
    lengths = torch.tensor([64, 1, 0, 17, 33, 2, 50, 63, 5], dtype=torch.int32, device="cuda")
    want, lse = zo.zo_cache_attend(q, kc, vc, table, lengths, lse=True)
    from paper_2609_38095_amd import decode
    work = torch.full((decode._lib().zo_cache_attend_work(9, 4, 2, 64),), 255, dtype=torch.uint8, device="cuda")  # NaN everywhere
    out = torch.zeros(9, 64, 4, device="cuda").transpose(1, 2).contiguous()
    wide_out = torch.zeros(9, 4, 80, device="cuda")
    for o in (out, wide_out[:, :, 3:67]):
        got = zo.zo_cache_attend(q, kc, vc, table, lengths, out=o, work=work)
        assert got.data_ptr() == o.data_ptr() and torch.equal(o, want)
    assert not wide_out[:, :, :3].any() and not wide_out[:, :, 67:].any()
    tokens = torch.full((3,), -5, dtype=torch.int32, device="cuda")
    logits, u = normal(1, (3, 100), "bf16"), torch.rand(3, device="cuda")
    assert zo.zo_draw(logits, u, tokens=tokens) is not None and torch.equal(tokens, zo.zo_draw(logits, u))
    assert zo.zo_draw(logits[:0], u[:0]).shape == (0,)
    assert zo.zo_cache_attend(q[:0], kc, vc, table[:0], lengths[:0]).shape == (0, 4, 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,vocab", [("peaked", 16_384), ("masked", 16_385), ("ties", 20_000), ("flat", 33_000), ("steep", 40_001),
                                        ("masked", 65_536), ("ties", 70_000), ("flat", 100_001), ("steep", 131_073),
                                        ("sorted", 151_936), ("peaked", (1 << 18) - 1)])
def test_draw_of_few_rows_is_that_of_many(kind, vocab, dtype):
    """Rows split over workgroups (few long ones) give what one workgroup for a row gives (the same rows repeated), and the oracle's
    tokens, where a part's list overflows too (ties, flat and sorted rows). The shorter rows are split without top-k only."""
    from paper_2609_38095_amd import decode
    settings = [  # temperature, top_k, top_p, min_p, u
        (1.0, 0, 1.0, 0.0, 0.5), (0.7, 0, 0.9, 0.0, 0.1), (1.3, 40, 1.0, 0.0, 0.99999994), (1.0, 512, 0.8, 0.0, 0.7),
        (1.0, 513, 0.9, 0.0, 0.9), (0.8, 0, 0.95, 0.01, 0.3), (1.0, 0, 1.0, 0.05, 0.6), (0.0, 0, 0.5, 0.0, 0.8),
        (1e30, 0, 0.5, 0.0, 0.5), (1e-30, 0, 0.5, 0.0, 0.5), (1.0, 1, 0.0, 0.0, 0.5), (1.0, 0, 0.0, 0.0, 0.99)]
    rows = len(settings)
    x = draw_rows("peaked" if kind == "sorted" else kind, rows, vocab, dtype, 3)
    if kind == "sorted":
        x = x.float().sort(dim=1, descending=True).values.to(x.dtype)
    counted = vocab >= 65_536
    need = decode._lib().zo_draw_work(rows, vocab, counted)
    assert need > 0 and decode._lib().zo_draw_work(4 * rows, vocab, counted) == 0
    t, k, p, m, u = (torch.tensor(c, dtype=torch.int32 if i == 1 else torch.float32, device="cuda") for i, c in enumerate(zip(*settings)))
    k, k_many = (k, k.repeat(4)) if counted else (None, None)
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    token, logprob = zo.zo_draw(x, u, t, k, p, m, logprobs=True, work=work)
    many = zo.zo_draw(x.repeat(4, 1), u.repeat(4), t.repeat(4), k_many, p.repeat(4), m.repeat(4), logprobs=True)
    again = zo.zo_draw(x, u, t, k, p, m, logprobs=True)
    for j in range(4):
        assert torch.equal(many[0][j * rows:(j + 1) * rows], token) and torch.equal(many[1][j * rows:(j + 1) * rows], logprob)
    assert torch.equal(again[0], token) and torch.equal(again[1], logprob)
    host = x.float().cpu().numpy()
    for b, (ti, ki, pi, mi, ui) in enumerate(settings):
        want, _ = oracle.draw(host[b], ui, ti, ki if counted else 0, pi, mi)
        assert int(token[b]) == want, (b, settings[b])
    with pytest.raises(zo.ZoError):
        zo.zo_draw(x, u, t, k, p, m, work=work[16:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_split_draw_on_a_stream_and_in_a_graph(dtype):
    """New logits and randoms in each replay, with eager draws between; no replay leans on what the workspace held."""
    x, u = draw_rows("peaked", 6, 50_272, dtype, 7), torch.rand(6, device="cuda")
    p = torch.tensor([0.9, 1.0, 0.3, 0.95, 0.0, 0.99], device="cuda")
    side = torch.cuda.Stream()
    want = zo.zo_draw(x, u, top_p=p, logprobs=True)
    torch.cuda.synchronize()
    got = zo.zo_draw(x, u, top_p=p, logprobs=True, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = zo.zo_draw(x, u, top_p=p, logprobs=True)
    for turn in range(4):
        x.copy_(draw_rows(("peaked", "steep", "ties", "masked")[turn], 6, 50_272, dtype, turn))
        u.copy_(torch.rand(6, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = zo.zo_draw(x.repeat(6, 1), u.repeat(6), top_p=p.repeat(6), logprobs=True)  # a workgroup for each row
        assert torch.equal(held[0], want[0][:6]) and torch.equal(held[1], want[1][:6])
