"""The operators of a decode step that takes several new tokens of each sequence at once, as cases
that can be timed and compared.

The new tokens of a sequence are a tree: drafted answers that share beginnings, or a chain (one
draft, or a prompt). A case is one call of one operator: the layout of the trees (which sequence a
token belongs to, its position, its place in the cache, which of the new tokens it sees), norm and
rotation of queries and keys with keys and values put at those places, attention of all new
tokens over the cache, the walk along the drafted tokens that the draws agree with, and the moves of
the walked path's keys and values to their final places. Head counts are those of `workloads`: OPT-1.3B
(32 heads of 64), OPT-13B (40 heads of 128), Qwen3-1.7B (16 query and 8 key heads of 128),
Qwen3-8B (32 and 8 of 128). Values are synthetic.

Where `own` is false, run() computes the operators in plain torch operations in 32 bits (angles
in 64); where it is true, it calls the library.

Fields of a case by op:
  lay      seqs, nodes (the most new tokens of a sequence), chain (no tree), context (the most cached tokens)
  put      dtype, seqs, nodes, q_heads, k_heads, dim, rotary, interleaved, norm, page, context
  attend   dtype, seqs, nodes, chain, q_heads, k_heads, dim, page, context, rows ("heads": a page holds its
           heads one after another, "tokens": its tokens)
  accept   seqs, nodes, chain, most (the longest path that is written)
  keep     dtype, layers, k_heads, dim, page, seqs, nodes, most
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6
BASE = 1e6
AT_ONCE = 1 << 27  # scores that the plain attention holds


def _lay(seqs, nodes, chain, context):
    return {"op": "lay", "seqs": seqs, "nodes": nodes, "chain": chain, "context": context}


def _put(dtype, seqs, nodes, heads, dim, rotary, page, context, interleaved=False, norm=True):
    return {"op": "put", "dtype": dtype, "seqs": seqs, "nodes": nodes, "q_heads": heads[0], "k_heads": heads[1], "dim": dim,
            "rotary": rotary, "interleaved": interleaved, "norm": norm, "page": page, "context": context, "chain": False}


def _attend(dtype, seqs, nodes, heads, dim, page, context, chain=False, rows="heads"):
    return {"op": "attend", "dtype": dtype, "seqs": seqs, "nodes": nodes, "chain": chain, "q_heads": heads[0], "k_heads": heads[1],
            "dim": dim, "page": page, "context": context, "rows": rows}


def _accept(seqs, nodes, chain, most):
    return {"op": "accept", "seqs": seqs, "nodes": nodes, "chain": chain, "most": most}


def _keep(dtype, layers, k_heads, dim, page, seqs, nodes, most):
    return {"op": "keep", "dtype": dtype, "layers": layers, "k_heads": k_heads, "dim": dim, "page": page, "seqs": seqs,
            "nodes": nodes, "most": most}


def listed():
    named = {
        # the layout of one answer's small draft, and of a batch of large trees: a step begins with it, so latency counts
        "lay_1_answer": _lay(1, 12, False, 1037),
        "lay_batch": _lay(256, 200, False, 4096),
        # a few drafted tokens of eight answers, and a batch of full trees, queries and keys from one fused projection
        "put_8_drafts": _put("bf16", 8, 6, (16, 8), 128, 128, 16, 2000),
        "put_batch": _put("bf16", 48, 64, (32, 8), 128, 128, 16, 4096),
        # one answer with a small draft over a short context
        "tree_1_answer": _attend("bf16", 1, 12, (32, 8), 128, 16, 1037),
        # a batch of trees over ragged contexts, pages that keep whole tokens together
        "tree_batch": _attend("bf16", 48, 64, (32, 8), 128, 16, 4096, rows="tokens"),
        # a key head for each query head, in 32 bits, an odd size of the trees
        "tree_f32_heads": _attend("f32", 16, 23, (32, 32), 64, 32, 2050),
        # prompts read at once behind what is cached of them: ragged chains, bound by the matrix products
        "prompts": _attend("bf16", 4, 6001, (32, 8), 128, 64, 2048, chain=True),
        # the walk of a few answers' trees, and of a batch's
        "accept_4_answers": _accept(4, 12, False, 8),
        "accept_batch": _accept(256, 200, False, 24),
        # a walked path brought together: one model's layers for a few answers, and for a batch
        "keep_8_answers": _keep("bf16", 28, 8, 128, 16, 8, 12, 8),
        "keep_batch": _keep("bf16", 36, 8, 128, 16, 256, 64, 16),
    }
    return [{"name": k, **v} for k, v in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("lay", "put", "attend", "attend", "attend", "accept", "keep"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    heads = rng.choice(((12, 12), (32, 32), (40, 40), (16, 8), (32, 8), (24, 4)))
    dim = rng.choice((64, 128, 128))
    page = rng.choice((16, 16, 32, 64, 128))
    flag = lambda p=0.5: rng.random() < p  # noqa: E731
    if op == "lay":
        return _lay(_log(rng, 1, 256), _log(rng, 1, 200), flag(0.3), _log(rng, 1, 30_000))
    if op == "put":
        return _put(dtype, _log(rng, 1, 48), _log(rng, 1, 64 if heads[0] + 2 * heads[1] <= 48 else 24), heads, dim,
                    rng.choice((dim, dim // 2)), page, _log(rng, 30, 3000), flag(), flag(0.7))
    if op == "attend":
        row = 2 * heads[1] * dim * SIZE[dtype]
        chain = flag(0.4)
        nodes = _log(rng, 1, 6000) if chain else _log(rng, 1, 120)
        context = _log(rng, 1, 40_000)
        # products, and bytes of the cache, of the largest listed case at most
        flops = 4 * dim * heads[0] * nodes * (context + nodes / 2)
        most = (1.5e12 if dtype == "bf16" else 1e11)
        while flops > most:
            nodes, context = (nodes + 1) // 2, (context + 1) // 2
            flops = 4 * dim * heads[0] * nodes * (context + nodes / 2)
        seqs = _log(rng, 1, max(1, min(96, 2 ** 30 // (row * (context + nodes)), int(most / flops))))
        return _attend(dtype, seqs, nodes, heads, dim, page, context, chain, rng.choice(("heads", "tokens")))
    if op == "accept":
        return _accept(_log(rng, 1, 256), _log(rng, 1, 200), flag(0.3), _log(rng, 1, 24))
    layers = rng.choice((1, 12, 24, 28, 36))
    return _keep(dtype, layers, heads[1], dim, page, _log(rng, 1, 256 if heads[1] <= 8 else 32), _log(rng, 2, 64), _log(rng, 2, 16))


# ---- what a program has in hand before the call

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, scale=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=g)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _ragged(n, longest, rng):
    """n counts up to the longest, the longest among them: the same ones for every seed, in another order."""
    got = np.maximum(1, (longest * np.sqrt((np.arange(n) + 0.5) / n)).astype(np.int64))
    got[-1] = longest
    return rng.permutation(got)


def _parents(nodes, rng):
    """For each node the one before it on its branch: half of them go on from the last one, the others branch off."""
    got = [-1]
    for i in range(1, nodes):
        got.append(i - 1 if rng.random() < 0.5 else int(rng.integers(i)))
    return got


def _depths(parents):
    got = []
    for p in parents:
        got.append(0 if p < 0 else got[p] + 1)
    return got


def _trees(case, rng, s):
    """The sequences' new tokens: where each sequence's begin, its cached tokens, and the trees on the host and the device."""
    counts = _ragged(case["seqs"], case["nodes"], rng)
    starts = np.concatenate(([0], np.cumsum(counts)))
    s["counts"], s["tokens"] = counts, int(starts[-1])
    s["starts"] = _dev(starts.astype(np.int32))
    trees = [list(range(-1, n - 1)) if case.get("chain") else _parents(n, rng) for n in counts.tolist()]
    s["depths"] = [_depths(t) for t in trees]
    s["deepest"] = max(max(d) for d in s["depths"])
    s["words"] = -(-case["nodes"] // 64)
    flat = np.concatenate([np.array(t, np.int32) for t in trees])
    s["parents"] = None if case.get("chain") else _dev(flat)
    s["trees"], s["starts_host"] = trees, starts
    if "context" in case:
        lengths = _ragged(case["seqs"], case["context"], rng)
        s["lengths_host"], s["lengths"] = lengths, _dev(lengths.astype(np.int32))


def _pages(case, context, counts, lengths, rng):
    """A page table over pages in scattered order, -1 past each sequence's end, and the number of pages: room for
    every sequence at the longest context with its new tokens."""
    width = -(-(context + case["nodes"]) // case["page"])
    need = -(-(lengths + counts) // case["page"])
    total = int((-(-(context + counts) // case["page"])).sum()) + 3
    order = rng.permutation(total).astype(np.int32)
    table, at = np.full((case["seqs"], width), -1, np.int32), 0
    for i, n in enumerate(need.tolist()):
        table[i, :n] = order[at:at + n]
        at += n
    return table, total


def _cache(case, g, pages):
    shape = (pages, case["k_heads"], case["page"], case["dim"])
    if case.get("rows") == "tokens":
        shape = (pages, case["page"], case["k_heads"], case["dim"])
        return [_normal(g, shape, DTYPES[case["dtype"]]).transpose(1, 2) for _ in range(2)]
    return [_normal(g, shape, DTYPES[case["dtype"]]) for _ in range(2)]


def _seen_words(trees, words):
    """Bit j of a token's words: it sees new token j of its sequence (itself and those before it on its branch)."""
    rows = []
    for tree in trees:
        bits = []
        for i, p in enumerate(tree):
            bits.append((bits[p] if p >= 0 else 0) | 1 << i)
        rows += [[(b >> (64 * w)) & (2 ** 64 - 1) for w in range(words)] for b in bits]
    return np.array(rows, np.uint64).reshape(-1, words).view(np.int64)


def _walk(tree, drafted, drawn, most):
    """The path from the first node along the drafted tokens that the draws agree with."""
    path = [0]
    while len(path) < most:
        after = [j for j, p in enumerate(tree) if p == path[-1] and drafted[j] == drawn[path[-1]]]
        if not after:
            break
        path.append(after[0])
    return path


def _tokens(s, rng):
    """Drafted tokens, siblings apart now and then, and draws that mostly agree with one of a node's children."""
    drafted, drawn = [], []
    for tree in s["trees"]:
        n = len(tree)
        a = rng.integers(0, 50_000, n)
        b = rng.integers(0, 50_000, n)
        for j, p in enumerate(tree):
            if p >= 0 and rng.random() < 0.6:
                b[p] = a[j]
        drafted.append(a)
        drawn.append(b)
    return drafted, drawn


def prepare(case, seed):
    g, rng = _gen(seed), np.random.default_rng(int(seed))
    s = dict(case)
    _trees(case, rng, s)
    if case["op"] == "put":
        hq, hk, d = case["q_heads"], case["k_heads"], case["dim"]
        x = _normal(g, (s["tokens"], hq + 2 * hk, d), DTYPES[case["dtype"]], 1.5)
        s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        s["q_gamma"], s["k_gamma"] = (None, None) if not case["norm"] else \
            tuple((1 + 0.1 * _normal(g, (d,), torch.float32)).to(DTYPES[case["dtype"]]) for _ in range(2))
        s["turns"] = BASE ** (-2.0 * np.arange(case["rotary"] // 2, dtype=np.float64) / case["rotary"]) / (2 * math.pi)
        seq = np.repeat(np.arange(case["seqs"]), s["counts"])
        s["seqs_of"] = _dev(seq.astype(np.int32))
        s["positions"] = _dev((s["lengths_host"][seq] + np.concatenate(s["depths"])).astype(np.int32))
        s["places"] = _dev((s["lengths_host"][seq] + np.arange(s["tokens"]) - s["starts_host"][seq]).astype(np.int32))
    if case["op"] in ("put", "attend"):
        table, pages = _pages(case, case["context"], s["counts"], s["lengths_host"], rng)
        s["table"] = _dev(table)
        s["k_cache"], s["v_cache"] = _cache(case, g, pages)
    if case["op"] == "attend":
        s["q"] = _normal(g, (s["tokens"], case["q_heads"], case["dim"]), DTYPES[case["dtype"]], 1.5)
        s["scale"] = case["dim"] ** -0.5
        s["seen"] = None if case["chain"] else _dev(_seen_words(s["trees"], s["words"]))
    if case["op"] == "accept":
        s["drafted_host"], s["drawn_host"] = _tokens(s, rng)
        s["drafted"], s["drawn"] = (_dev(np.concatenate(s[n]).astype(np.int32)) for n in ("drafted_host", "drawn_host"))
    if case["op"] == "keep":
        drafted, drawn = _tokens(s, rng)
        path = np.full((case["seqs"], case["most"]), -1, np.int32)
        for i, tree in enumerate(s["trees"]):
            at = _walk(tree, drafted[i], drawn[i], case["most"])
            path[i, :len(at)] = at
        s["path"], s["path_host"] = _dev(path), path
        lengths = rng.integers(0, 4 * case["page"], case["seqs"])
        s["lengths"], s["lengths_host"] = _dev(lengths.astype(np.int32)), lengths
        table, pages = _pages(case, 4 * case["page"], s["counts"], lengths, rng)
        s["table"] = _dev(table)
        s["cache"] = _normal(g, (case["layers"], 2, pages, case["k_heads"], case["page"], case["dim"]), DTYPES[case["dtype"]])
        s["k_caches"] = [s["cache"][i, 0] for i in range(case["layers"])]
        s["v_caches"] = [s["cache"][i, 1] for i in range(case["layers"])]
    return s


# ---- the plain forms

def _seq_of(s):
    token = torch.arange(s["tokens"], device="cuda")
    starts = s["starts"].long()
    seq = torch.searchsorted(starts[1:], token, right=True)
    return token, starts, seq, token - starts[seq]


def _plain_lay(s):
    token, starts, seq, i = _seq_of(s)
    places = s["lengths"].long()[seq] + i
    if s["parents"] is None:
        return seq.int(), places.int(), places.int()
    parents, word = s["parents"].long(), torch.arange(s["words"], device="cuda")[None]
    at, depth = i, torch.full_like(i, -1)
    seen = torch.zeros((s["tokens"], s["words"]), dtype=torch.int64, device="cuda")
    one = torch.ones((), dtype=torch.int64, device="cuda")
    for _ in range(s["deepest"] + 1):
        live = at >= 0
        bit = torch.bitwise_left_shift(one, at.clamp(min=0) % 64)[:, None]
        seen |= torch.where(live[:, None] & (at[:, None] // 64 == word), bit, 0)
        depth += live
        at = torch.where(live, parents[starts[seq] + at.clamp(min=0)], -1)
    return seq.int(), (s["lengths"].long()[seq] + depth).int(), places.int(), seen


def _turn(x, s):
    """Rotates the first dims of each row of x by its token's angles."""
    turns = torch.from_numpy(s["turns"]).cuda()
    angle = torch.remainder(s["positions"].double()[:, None] * turns, 1.0).float() * (2 * math.pi)
    cos, sin, r = torch.cos(angle)[:, None], torch.sin(angle)[:, None], s["rotary"]
    if s["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((y, x[..., r:]), dim=-1)


def _forward(x, gamma, s):
    y = x.float()
    if gamma is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gamma.float()
    return _turn(y, s).to(x.dtype)


def _plain_put(s):
    q, k = (_forward(s[n], s[n + "_gamma"], s) for n in "qk")
    at = s["places"].long()
    page = s["table"][s["seqs_of"].long(), at // s["page"]].long()
    s["k_cache"][page, :, at % s["page"]] = k
    s["v_cache"][page, :, at % s["page"]] = s["v"]
    return q, s["k_cache"], s["v_cache"]


def _attend_some(s, seqs, heads, out, lse):
    """The attention of some sequences' tokens, padded to the longest of them, for some key heads."""
    group, d = s["q_heads"] // s["k_heads"], s["dim"]
    counts = s["counts"][seqs]
    n = int(counts.max())
    width = -(-int((s["lengths_host"][seqs] + counts).max()) // s["page"])
    starts, lengths = s["starts"].long()[:-1][seqs], s["lengths"].long()[seqs]
    count = s["starts"].long()[1:][seqs] - starts
    i = torch.arange(n, device="cuda")
    token = (starts[:, None] + i).clamp(max=s["tokens"] - 1)  # [sequences, n]
    ids = s["table"][seqs, :width].clamp(min=0).long()
    b, h = ids.shape[0], heads.stop - heads.start
    k, v = (c[:, heads][ids].permute(0, 2, 1, 3, 4).reshape(b, h, -1, d).float() for c in (s["k_cache"], s["v_cache"]))
    j = torch.arange(width * s["page"], device="cuda")[None, None] - lengths[:, None, None]  # of the new tokens
    if s["seen"] is None:
        live = j <= i[None, :, None]
    else:
        e = j.clamp(min=0).expand(b, n, -1)
        words = torch.gather(s["seen"][token], 2, (e // 64).clamp(max=s["words"] - 1))
        live = (j < 0) | ((torch.bitwise_right_shift(words, e % 64) & 1) != 0) & (e < 64 * s["words"])
    live = live & (j < count[:, None, None])
    live = live.repeat_interleave(group, 1)[:, None]  # [sequences, 1, n group, keys]
    q = s["q"][token].reshape(b, n, s["k_heads"], group, d)[:, :, heads]
    q = q.permute(0, 2, 1, 3, 4).reshape(b, h, n * group, d).float() * s["scale"]
    score = torch.where(live, torch.matmul(q, k.transpose(2, 3)), -math.inf)
    top = score.amax(-1, keepdim=True)
    score = torch.exp(score - top)
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score, v) / total
    o = o.reshape(b, h, n, group, d).transpose(1, 2)
    sums = (top + torch.log(total)).reshape(b, h, n, group).transpose(1, 2)
    there = i[None] < count[:, None]
    at = slice(heads.start * group, heads.stop * group)
    out[token[there], at] = o[there].reshape(-1, h * group, d).to(out.dtype)
    lse[token[there], at] = sums[there].reshape(-1, h * group)


def _plain_attend(s):
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], device="cuda")
    scores = int(s["counts"].max()) * s["q_heads"] * int((s["lengths_host"] + s["counts"]).max())
    if scores * s["seqs"] <= AT_ONCE:
        _attend_some(s, slice(0, s["seqs"]), slice(0, s["k_heads"]), out, lse)
    else:
        each = max(1, AT_ONCE // scores)
        heads = max(1, min(s["k_heads"], s["k_heads"] * AT_ONCE // scores))
        for i in range(0, s["seqs"], each):
            for h in range(0, s["k_heads"], heads):
                _attend_some(s, slice(i, min(i + each, s["seqs"])), slice(h, min(h + heads, s["k_heads"])), out, lse)
    return out, lse


def _plain_accept(s):
    starts, n = s["starts"].long(), int(s["counts"].max())
    i = torch.arange(n, device="cuda")[None]
    token = (starts[:-1, None] + i).clamp(max=s["tokens"] - 1)
    there = i < (starts[1:] - starts[:-1])[:, None]
    parents = (i - 1).expand(s["seqs"], n) if s["parents"] is None else s["parents"].long()[token]
    drafted, drawn = s["drafted"].long()[token], s["drawn"].long()[token]
    at = torch.zeros((s["seqs"], 1), dtype=torch.int64, device="cuda")
    path, tokens = [], []
    for _ in range(s["most"]):
        said = torch.where(at >= 0, torch.gather(drawn, 1, at.clamp(min=0)), -1)
        path.append(at)
        tokens.append(said)
        after = there & (parents == at) & (drafted == said) & (at >= 0)
        at = torch.where(after, i, n).amin(1, keepdim=True)
        at = torch.where(at < n, at, -1)
    path, tokens = torch.cat(path, 1), torch.cat(tokens, 1)
    return path.int(), tokens.int(), (path >= 0).sum(1).int()


def _plain_keep(s):
    path = s["path"].long()
    seq, i = torch.nonzero(path >= 0, as_tuple=True)
    lengths = s["lengths"].long()[seq]
    src, dst = lengths + path[seq, i], lengths + i
    page = s["page"]
    a, b = (s["table"][seq, at // page].long() for at in (src, dst))
    c = s["cache"].flatten(0, 1)
    c[:, b, :, dst % page] = c[:, a, :, src % page]
    return s["cache"]


# ---- the library's calls

def _own(s):
    import paper_2609_38095_amd as zo
    if s["op"] == "lay":
        seqs, positions, places, seen = zo.zo_tree_lay(s["starts"], s["lengths"], s["tokens"], s["parents"], s["words"] if s["parents"] is not None else 0)
        return (seqs, positions, places) if seen is None else (seqs, positions, places, seen)
    if s["op"] == "put":
        q = zo.zo_norm_rotate_put(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["positions"], s["turns"],
                                  interleaved=s["interleaved"], q_gamma=s["q_gamma"], k_gamma=s["k_gamma"], norm_eps=EPS,
                                  seqs=s["seqs_of"], places=s["places"])
        return q, s["k_cache"], s["v_cache"]
    if s["op"] == "attend":
        return zo.zo_tree_attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["starts"], seen=s["seen"],
                                 scale=s["scale"], lse=True)
    if s["op"] == "accept":
        return zo.zo_tree_accept(s["drafted"], s["drawn"], s["starts"], s["most"], parents=s["parents"])
    zo.zo_tree_keep(s["k_caches"], s["v_caches"], s["table"], s["lengths"], s["path"])
    return s["cache"]


def run(state):
    if own:
        return _own(state)
    return {"lay": _plain_lay, "put": _plain_put, "attend": _plain_attend, "accept": _plain_accept, "keep": _plain_keep}[state["op"]](state)


# ---- the least work, and the definitions in 64 bits

def work(case):
    mean = lambda most: most * (1 + (case["seqs"] - 1) * 2 / 3)  # noqa: E731 (the sum of the ragged counts, about)
    tokens = mean(case["nodes"])
    if case["op"] == "lay":
        words = 0 if case["chain"] else -(-case["nodes"] // 64)
        return {"bytes": tokens * (12 + 8 * words + (0 if case["chain"] else 4)) + 8 * case["seqs"], "flops": tokens}
    if case["op"] == "put":
        n = tokens * (case["q_heads"] + 2 * case["k_heads"]) * case["dim"]
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 12 * tokens, "flops": n * (4 * case["norm"] + 3)}
    if case["op"] == "attend":
        size, d, cached = SIZE[case["dtype"]], case["dim"], mean(case["context"])
        seen = case["nodes"] / 3 if case["chain"] else 4  # of the new tokens, by each of them
        return {"bytes": (cached + tokens) * case["k_heads"] * d * 2 * size + 2 * tokens * case["q_heads"] * d * size,
                "flops": 4 * tokens * case["q_heads"] * d * (cached / case["seqs"] + seen)}
    if case["op"] == "accept":
        return {"bytes": tokens * (8 if case["chain"] else 12) + case["seqs"] * (8 * case["most"] + 8), "flops": tokens}
    # about two rows of a path move
    row = 2 * case["layers"] * case["k_heads"] * case["dim"] * SIZE[case["dtype"]]
    return {"bytes": case["seqs"] * (2 * 2 * row + 4 * case["most"]), "flops": 0}


def _exact_lay(case, s):
    seqs, positions, places, seen = [], [], [], []
    for i, tree in enumerate(s["trees"]):
        for j in range(len(tree)):
            branch, at = [], j
            while at >= 0:
                branch.append(at)
                at = tree[at]
            seqs.append(i)
            positions.append(int(s["lengths_host"][i]) + len(branch) - 1)
            places.append(int(s["lengths_host"][i]) + j)
            seen.append([np.array(sum(1 << (b % 64) for b in branch if b // 64 == w), np.uint64) for w in range(s["words"])]
                        if not case["chain"] else [])
    got = tuple(np.array(x, np.int32) for x in (seqs, positions, places))
    return got if case["chain"] else got + (np.array(seen, np.uint64).view(np.int64).reshape(-1, s["words"]),)


def _exact_rows(case, x, gamma, s):
    """The definition with complex numbers: a pair is one of them, a position a factor of modulus one."""
    if gamma is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS) * gamma.double()
    r = case["rotary"]
    head = x[..., :r]
    pairs = head.reshape(*head.shape[:-1], r // 2, 2) if case["interleaved"] else \
        head.reshape(*head.shape[:-1], 2, r // 2).transpose(-1, -2)
    z = torch.complex(pairs[..., 0], pairs[..., 1])
    turned = torch.outer(s["positions"].double(), torch.from_numpy(s["turns"]).cuda())
    z = z * torch.polar(torch.ones_like(turned), 2 * math.pi * (turned - torch.floor(turned)))[:, None]
    parts = torch.view_as_real(z)
    parts = parts if case["interleaved"] else parts.transpose(-1, -2)
    return torch.cat((parts.reshape(head.shape), x[..., r:]), dim=-1)


def _exact_put(case, s):
    q, k = (_exact_rows(case, s[n].double(), s[n + "_gamma"], s) for n in "qk")
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    t = 0
    for i, n in enumerate(s["counts"].tolist()):
        for at in range(int(s["lengths_host"][i]), int(s["lengths_host"][i]) + n):
            page = int(s["table"][i, at // case["page"]])
            k_cache[page, :, at % case["page"]] = k[t]
            v_cache[page, :, at % case["page"]] = s["v"][t].double()
            t += 1
    return q, k_cache, v_cache


def _exact_attend(case, s):
    group, d = case["q_heads"] // case["k_heads"], case["dim"]
    out = torch.empty((s["tokens"], case["q_heads"], d), dtype=torch.float64, device="cuda")
    lse = torch.empty((s["tokens"], case["q_heads"]), dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["counts"].tolist()):
        cached, first = int(s["lengths_host"][i]), int(s["starts_host"][i])
        if case["chain"]:
            branch = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        else:
            rows = np.zeros((n, n), bool)
            for j, p in enumerate(s["trees"][i]):
                if p >= 0:
                    rows[j] = rows[p]
                rows[j, j] = True
            branch = _dev(rows)
        hidden = torch.cat((torch.zeros(n, cached, dtype=torch.bool, device="cuda"), ~branch), 1)[:, None]
        pages = s["table"][i, :-(-(cached + n) // case["page"])].long()
        for h in range(case["k_heads"]):
            k, v = (c[pages, h].reshape(-1, d)[:cached + n].double() for c in (s["k_cache"], s["v_cache"]))
            heads = slice(h * group, (h + 1) * group)
            q = s["q"][first:first + n, heads].double().reshape(n * group, d)
            score = (q @ k.T.contiguous() * s["scale"]).reshape(n, group, -1).masked_fill(hidden, -math.inf)
            sums = torch.logsumexp(score, -1, keepdim=True)
            weights = torch.exp(score - sums).reshape(n * group, -1)
            out[first:first + n, heads] = (weights @ v).reshape(n, group, d)
            lse[first:first + n, heads] = sums[..., 0]
    return out, lse


def _exact_accept(case, s):
    path = np.full((case["seqs"], case["most"]), -1, np.int32)
    tokens, counts = path.copy(), np.zeros(case["seqs"], np.int32)
    for i, tree in enumerate(s["trees"]):
        at = _walk(tree, s["drafted_host"][i], s["drawn_host"][i], case["most"])
        path[i, :len(at)], counts[i] = at, len(at)
        tokens[i, :len(at)] = s["drawn_host"][i][at]
    return path, tokens, counts


def exact(case, seed):
    if case["op"] == "keep":
        return None  # nothing is computed
    s = prepare(case, seed)
    return {"lay": _exact_lay, "put": _exact_put, "attend": _exact_attend, "accept": _exact_accept}[case["op"]](case, s)
