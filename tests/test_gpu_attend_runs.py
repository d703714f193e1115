"""zo_cache_attend where a wave's run of tiles is long: several tiles of a sequence, whole sequences inside a run, runs that begin
and end inside sequences, page ids looked up more than once. The oracle is torch in float64 on the GPU.

Tolerances, with e = 2^-24: a score is a sum of dim products, off by at most (dim + 8) e of the sum of their magnitudes, which
moves each weight by that share, twice (weight and sum); sums add a rounding for each 16 tokens and 64 for joins and rescalings, and
a bf16 weight meets its value as two parts (2^-16, 2^8 e); a bf16 result adds half an ulp."""

import math

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def tiles_and_waves(lengths, q_heads, heads, dim, dtype):
    """Tiles of a call, and the waves that they are dealt out to at most."""
    tile = 32 if dtype == "bf16" else 16
    items = heads * -(-(q_heads // heads) // 16)
    return sum(-(-n // tile) for n in lengths) * items, 1024 * (2 if dim > 128 else 3 if dim > 64 else 4)


def setup(lengths, q_heads, heads, dim, page, dtype, seed, rows="heads"):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    width, pages = max(need), sum(need) + 3
    ids, at = rng.permutation(pages).astype(np.int32), 0
    table = np.full((len(lengths), width), -1, np.int32)
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n]
        at += n
    normal = lambda *shape: torch.empty(shape, device="cuda").normal_(generator=g).to(TYPES[dtype])  # noqa: E731
    if rows == "heads":
        k, v = (normal(pages, heads, page, dim) for _ in range(2))
    else:
        k, v = (normal(pages, page, heads, dim).transpose(1, 2) for _ in range(2))
    return normal(len(lengths), q_heads, dim), k, v, torch.from_numpy(table).cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")


def tokens_of(cache, row, n, page):
    """[heads, n, dim] of a sequence, in float64."""
    return cache[row[:-(-n // page)].long()].transpose(0, 1).flatten(1, 2)[:, :n].double()


def compare(q, k, v, table, lengths, page, scale, dtype):
    out, lse = zo.zo_cache_attend(q, k, v, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), scale, lse=True)
    heads, dim = k.shape[1], q.shape[2]
    for s, n in enumerate(lengths):
        if n == 0:
            assert not out[s].any() and bool((lse[s] == -math.inf).all())
            continue
        kk, vv = tokens_of(k, table[s], n, page), tokens_of(v, table[s], n, page)
        qq = q[s].double().view(heads, -1, dim)
        x = scale * (qq @ kk.transpose(1, 2).contiguous())
        big = abs(scale) * (qq.abs() @ kk.abs().transpose(1, 2).contiguous()).amax(2, keepdim=True)
        p = torch.softmax(x, 2)
        want, magnitude, want_lse = p @ vv, p @ vv.abs(), torch.logsumexp(x, 2)
        steps = 2 * (dim + 8) * big + n / 16 + 64 + (2 ** 8 if dtype == "bf16" else 0)
        half_ulp = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=1e-38))) - 8) if dtype == "bf16" else 0.0
        off = (out[s].double().view_as(want) - want).abs() / (steps * E * magnitude + half_ulp + 1e-37)
        assert float(off.max()) <= 1.0, (s, n, float(off.max()))
        off = (lse[s].double().view(heads, -1) - want_lse).abs() / ((steps[..., 0] + 8 * want_lse.abs()) * E)
        assert float(off.max()) <= 1.0, (s, n, float(off.max()))
    assert torch.equal(out, zo.zo_cache_attend(q, k, v, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), scale))


FORMS = [  # q heads, k heads, dim, page, layout: the matrix-core forms and (by size of head or page) the element-wise ones
    (8, 8, 64, 16, "heads"), (16, 8, 128, 16, "tokens"), (16, 8, 128, 48, "heads"), (8, 8, 256, 64, "heads"),
    (20, 1, 128, 32, "heads"), (8, 8, 80, 16, "heads"), (8, 8, 64, 7, "tokens"), (8, 4, 200, 24, "heads")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", FORMS, ids=[str(i) for i in range(len(FORMS))])
def test_many_ragged_sequences(form, dtype):
    """Runs that begin and end inside sequences, with short sequences between."""
    hq, hk, dim, page, rows = form
    rng = np.random.default_rng(dim + page)
    lengths = np.where(rng.random(300) < 0.3, rng.integers(0, 40, 300), rng.integers(0, 1500, 300))
    lengths[[0, 7, 299]] = [0, 1, 1500]
    lengths = np.concatenate([lengths] * (1 if hk == 8 else 2 if hk == 4 else 4)).tolist()
    tiles, waves = tiles_and_waves(lengths, hq, hk, dim, dtype)
    assert tiles > 2 * waves
    q, k, v, table, _ = setup(lengths, hq, hk, dim, page, dtype, dim, rows)
    compare(q, k, v, table, lengths, page, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", FORMS, ids=[str(i) for i in range(len(FORMS))])
def test_few_long_sequences(form, dtype):
    """More than 64 sixteens of tokens for a wave, so that a run looks page ids up more than once; parts of many workgroups."""
    hq, hk, dim, page, rows = form
    per = 1024 * (2 if dim > 128 else 3 if dim > 64 else 4) * 72 * 16 // (hk * -(-hq // hk // 16))  # tokens: 72 sixteens a wave
    lengths = [per // 2 + 5, 3, per // 2 + 1111]
    tiles, waves = tiles_and_waves(lengths, hq, hk, dim, dtype)
    assert tiles * (2 if dtype == "bf16" else 1) > 64 * waves
    q, k, v, table, _ = setup(lengths, hq, hk, dim, page, dtype, dim, rows)
    compare(q, k, v, table, lengths, page, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", FORMS, ids=[str(i) for i in range(len(FORMS))])
def test_scores_that_rise_along_a_sequence(form, dtype):
    """The bound of the scores is raised again and again within a run, in one head while others stay as they are."""
    hq, hk, dim, page, rows = form
    rng = np.random.default_rng(1)
    lengths = rng.integers(100, 900, 300 if hk == 8 else 600 if hk == 4 else 1200).tolist()
    tiles, waves = tiles_and_waves(lengths, hq, hk, dim, dtype)
    assert tiles > 2 * waves
    q, k, v, table, _ = setup(lengths, hq, hk, dim, page, dtype, 3, rows)
    q[..., 0] = 1.0
    q[:, ::3, 0] = -1.0  # falling scores
    q[:, 1::3, 0] = 0.0  # neither
    at = torch.arange(max(lengths), device="cuda")
    rise = (0.5 * (at // 4)).to(k.dtype)  # 0.5 for each 4 tokens: 4 and 2 for a tile
    for s, n in enumerate(lengths):
        ids = table[s, :-(-n // page)].long()
        k[ids, :, :, 0] = torch.cat((rise[:n], rise.new_zeros(len(ids) * page - n))).view(len(ids), 1, page).expand(-1, hk, -1)
    compare(q, k, v, table, lengths, page, 1.0, dtype)
