"""The operators of a decode step, as cases that can be timed and compared.

A case is one call of one operator: the head norms and position rotation of queries and keys
(forward, backward, and the form that puts the new keys and values in a paged cache), the
attention of one new token per sequence over the cache, the copying of cache pages, and the
draw of a token from logits. Head counts and vocabularies are those of `workloads`: OPT-1.3B
(32 heads of 64), OPT-13B (40 heads of 128), Qwen3-1.7B (16 query and 8 key heads of 128),
Qwen3-8B (32 and 8 of 128). Values are synthetic.

Where `own` is false, run() computes the operators in plain torch operations in 32 bits
(angles, and weights whose sums decide a whole number, in 64); where it is true, it calls the
library.

Fields of a case by op:
  rotate, rotate_back   dtype, tokens, q_heads, k_heads, dim, rotary (rotated dims), interleaved,
                        norm, fused (queries, keys and values are views of one projection), far
                        (the positions' range)
  rotate_put            dtype, seqs, q_heads, k_heads, dim, rotary, interleaved, norm, page, longest
  attend                dtype, seqs, q_heads, k_heads, dim, page, longest, empty (share of empty
                        sequences), rows ("heads": a page holds its heads one after another,
                        "tokens": its tokens)
  copy                  dtype, layers, k_heads, dim, page, pairs, full (whole pages, else ragged)
  draw                  dtype, seqs, vocab, top_k, top_p, min_p (the largest values in the batch)
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6
BASE = 1e6
ONE = 1 << 44  # the weight of the largest logit


def _rotate(op, dtype, tokens, heads, dim, rotary, interleaved=False, norm=True, fused=True, far=4096):
    return {"op": op, "dtype": dtype, "tokens": tokens, "q_heads": heads[0], "k_heads": heads[1], "dim": dim,
            "rotary": rotary, "interleaved": interleaved, "norm": norm, "fused": fused, "far": far}


def _put(dtype, seqs, heads, dim, rotary, page, longest, interleaved=False, norm=True):
    return {"op": "rotate_put", "dtype": dtype, "seqs": seqs, "q_heads": heads[0], "k_heads": heads[1], "dim": dim,
            "rotary": rotary, "interleaved": interleaved, "norm": norm, "page": page, "longest": longest}


def _attend(dtype, seqs, heads, dim, page, longest, empty=0.0, rows="heads"):
    return {"op": "attend", "dtype": dtype, "seqs": seqs, "q_heads": heads[0], "k_heads": heads[1], "dim": dim,
            "page": page, "longest": longest, "empty": empty, "rows": rows}


def _copy(dtype, layers, k_heads, dim, page, pairs, full):
    return {"op": "copy", "dtype": dtype, "layers": layers, "k_heads": k_heads, "dim": dim, "page": page,
            "pairs": pairs, "full": full}


def _draw(dtype, seqs, vocab, top_k, top_p, min_p):
    return {"op": "draw", "dtype": dtype, "seqs": seqs, "vocab": vocab, "top_k": top_k, "top_p": top_p, "min_p": min_p}


def listed():
    named = {
        # one decode step of eight answers: a few rows, where a call's latency counts
        "put_8_answers": _put("bf16", 8, (16, 8), 128, 128, 16, 2000),
        # the queries and keys of a packed batch of prompts, views of one fused projection
        "rotate_prompts": _rotate("rotate", "bf16", 4096, (32, 8), 128, 128),
        # 32-bit weights, pairs side by side, half of each head rotated, no norm, an odd count of tokens
        "rotate_f32_part": _rotate("rotate", "f32", 16387, (32, 32), 64, 32, interleaved=True, norm=False, fused=False,
                                   far=100_000),
        # the gradient of a long batch
        "rotate_back_batch": _rotate("rotate_back", "bf16", 8192, (32, 8), 128, 128),
        # one answer growing: a single short sequence
        "attend_1_answer": _attend("bf16", 1, (32, 8), 128, 16, 1037),
        # a batch of answers of ragged lengths, pages that keep whole tokens together
        "attend_batch": _attend("bf16", 48, (32, 8), 128, 16, 4096, rows="tokens"),
        # few sequences over a long context
        "attend_long": _attend("bf16", 4, (16, 8), 128, 64, 131_072),
        # a key head for each query head, in 32 bits, some sequences still empty
        "attend_f32_heads": _attend("f32", 16, (32, 32), 64, 32, 2050, empty=0.2),
        # several answers forked from their prompts: the partly filled last page of each, every layer
        "fork_32_answers": _copy("bf16", 28, 8, 128, 16, 32, False),
        # a cache brought together: whole pages moved down, every layer
        "compact_pages": _copy("bf16", 28, 8, 128, 16, 1024, True),
        # the tokens of a few answers, and of a large batch of samples
        "draw_4_answers": _draw("f32", 4, 151_936, 50, 0.9, 0.0),
        "draw_batch": _draw("bf16", 256, 151_936, 0, 0.95, 0.02),
    }
    return [{"name": k, **v} for k, v in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotate", "rotate_back", "rotate_put", "attend", "attend", "copy", "draw"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    heads = rng.choice(((12, 12), (32, 32), (40, 40), (16, 8), (32, 8), (24, 4)))
    dim = rng.choice((64, 128, 128))
    rotary = rng.choice((dim, dim // 2))
    flag = lambda: rng.random() < 0.5  # noqa: E731
    page = rng.choice((16, 16, 32, 64, 128))
    if op in ("rotate", "rotate_back"):
        most = 2 ** 27 // ((heads[0] + heads[1]) * dim * SIZE[dtype])
        return _rotate(op, dtype, _log(rng, 1, most), heads, dim, rotary, flag(), rng.random() < 0.7, flag(), _log(rng, 1000, 200_000))
    if op == "rotate_put":
        return _put(dtype, _log(rng, 1, 512), heads, dim, rotary, page, _log(rng, 30, 3000), flag(), rng.random() < 0.7)
    if op == "attend":
        row = 2 * heads[1] * dim * SIZE[dtype]
        longest = _log(rng, 1, 60_000)
        seqs = _log(rng, 1, max(1, min(300, 2 ** 30 // (row * longest))))
        return _attend(dtype, seqs, heads, dim, page, longest, rng.choice((0.0, 0.0, 0.3)), rng.choice(("heads", "tokens")))
    if op == "copy":
        layers = rng.choice((1, 12, 24, 28, 36))
        row = 2 * layers * heads[1] * dim * page * SIZE[dtype]
        return _copy(dtype, layers, heads[1], dim, page, _log(rng, 1, max(1, min(2000, 2 ** 30 // row))), flag())
    vocab = rng.choice((50_272, 151_936, 32_001, 1009))
    return _draw(dtype, _log(rng, 1, 200), vocab, rng.choice((0, 1, 20, 200)), rng.choice((1.0, 0.9, 0.95, 0.5)),
                 rng.choice((0.0, 0.0, 0.05)))


# ---- what a program has in hand before the call

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, scale=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=g)


def _lengths(case, rng):
    """Ragged lengths up to the longest, the longest among them."""
    n = case["seqs"]
    got = np.maximum(1, (case["longest"] * np.sqrt(rng.random(n))).astype(np.int64))
    got[rng.integers(n)] = case["longest"]
    if case.get("empty"):
        got[rng.random(n) < case["empty"]] = 0
    return got


def _pages(case, lengths, rng):
    """A page table over pages in scattered order, -1 past each sequence's end, and the number of
    pages: room for every sequence at the longest length."""
    width = -(-case["longest"] // case["page"])
    total = case["seqs"] * width + 3
    order = rng.permutation(total).astype(np.int32)[:case["seqs"] * width].reshape(case["seqs"], width)
    need = -(-lengths // case["page"])
    return np.where(np.arange(width)[None] < need[:, None], order, -1).astype(np.int32), total


def _cache(case, g, pages):
    shape = (pages, case["k_heads"], case["page"], case["dim"])
    if case.get("rows") == "tokens":
        shape = (pages, case["page"], case["k_heads"], case["dim"])
        return [_normal(g, shape, DTYPES[case["dtype"]]).transpose(1, 2) for _ in range(2)]
    return [_normal(g, shape, DTYPES[case["dtype"]]) for _ in range(2)]


def _qkv(case, g, tokens, fused):
    hq, hk, d = case["q_heads"], case["k_heads"], case["dim"]
    if fused:
        x = _normal(g, (tokens, hq + 2 * hk, d), DTYPES[case["dtype"]], 1.5)
        return x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    return tuple(_normal(g, (tokens, h, d), DTYPES[case["dtype"]], 1.5) for h in (hq, hk, hk))


def _gammas(case, g):
    if not case["norm"]:
        return None, None
    return tuple((1 + 0.1 * _normal(g, (case["dim"],), torch.float32)).to(DTYPES[case["dtype"]]) for _ in range(2))


def _turns(case):
    i = np.arange(case["rotary"] // 2, dtype=np.float64)
    return BASE ** (-2.0 * i / case["rotary"]) / (2 * math.pi)


def prepare(case, seed):
    g, rng = _gen(seed), np.random.default_rng(int(seed))
    s = dict(case)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    if case["op"] in ("rotate", "rotate_back"):
        n = case["tokens"]
        s["q"], s["k"], _ = _qkv(case, g, n, case["fused"])
        s["q_gamma"], s["k_gamma"] = _gammas(case, g)
        s["turns"] = _turns(case)
        at = (np.arange(n) + rng.integers(case["far"])) % case["far"]  # documents packed one after another
        s["positions"] = dev(at.astype(np.int32))
        if case["op"] == "rotate_back":
            s["dq_out"] = _normal(g, (n, case["q_heads"], case["dim"]), DTYPES[case["dtype"]])
            s["dk_out"] = _normal(g, (n, case["k_heads"], case["dim"]), DTYPES[case["dtype"]])
    elif case["op"] == "rotate_put":
        lengths = _lengths(case, rng)
        table, pages = _pages(case, lengths, rng)
        s["q"], s["k"], s["v"] = _qkv(case, g, case["seqs"], True)
        s["q_gamma"], s["k_gamma"] = _gammas(case, g)
        s["turns"] = _turns(case)
        s["k_cache"], s["v_cache"] = _cache(case, g, pages)
        s["table"], s["positions"] = dev(table), dev((lengths - 1).astype(np.int32))
    elif case["op"] == "attend":
        lengths = _lengths(case, rng)
        table, pages = _pages(case, lengths, rng)
        s["k_cache"], s["v_cache"] = _cache(case, g, pages)
        s["q"] = _normal(g, (case["seqs"], case["q_heads"], case["dim"]), DTYPES[case["dtype"]], 1.5)
        s["table"], s["lengths"] = dev(table), dev(lengths.astype(np.int32))
        s["scale"] = case["dim"] ** -0.5
    elif case["op"] == "copy":
        n, page = case["pairs"], case["page"]
        pages = 2 * n + 8
        s["cache"] = _normal(g, (case["layers"], 2, pages, case["k_heads"], page, case["dim"]), DTYPES[case["dtype"]])
        s["k_caches"] = [s["cache"][i, 0] for i in range(case["layers"])]
        s["v_caches"] = [s["cache"][i, 1] for i in range(case["layers"])]
        order = rng.permutation(pages)
        s["src"], s["dst"] = order[:n].astype(np.int32), order[n:2 * n].astype(np.int32)
        s["rows"] = np.full(n, page, np.int32) if case["full"] else rng.integers(1, page + 1, n).astype(np.int32)
    else:
        n, v = case["seqs"], case["vocab"]
        # logits of a language model: a wide bulk, and a few tokens well above it
        x = _normal(g, (n, v), torch.float32, 2.0)
        heads = min(64, v // 4)
        at = torch.randint(0, v, (n, heads), generator=g, device="cuda")
        x.scatter_(1, at, _normal(g, (n, heads), torch.float32, 2.0) + 9.0)
        s["logits"] = x.to(DTYPES[case["dtype"]])
        s["u"] = torch.rand(n, generator=g, device="cuda")
        s["temperature"] = dev(rng.uniform(0.5, 1.2, n).astype(np.float32))
        s["top_k"] = dev(np.where(rng.random(n) < 0.8, case["top_k"], 0).astype(np.int32)) if case["top_k"] else None
        s["top_p"] = dev(rng.uniform(0.8 * case["top_p"], case["top_p"], n).astype(np.float32)) if case["top_p"] < 1 else None
        s["min_p"] = dev(rng.uniform(0, case["min_p"], n).astype(np.float32)) if case["min_p"] else None
    return s


# ---- the plain forms

def _cos_sin(s):
    turns = torch.from_numpy(s["turns"]).cuda()
    angle = torch.remainder(s["positions"].double()[:, None] * turns, 1.0).float() * (2 * math.pi)
    return torch.cos(angle)[:, None], torch.sin(angle)[:, None]


def _turn(x, cos, sin, s):
    """Rotates the first dims of each row of x by the angles."""
    r = s["rotary"]
    if s["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((y, x[..., r:]), dim=-1)


def _forward(x, gamma, cos, sin, s):
    y = x.float()
    if gamma is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gamma.float()
    return torch.where((s["positions"] >= 0)[:, None, None], _turn(y, cos, sin, s), 0.0).to(x.dtype)


def _backward(dy, x, gamma, cos, sin, s):
    dn = torch.where((s["positions"] >= 0)[:, None, None], _turn(dy.float(), cos, -sin, s), 0.0)
    if gamma is None:
        return dn.to(x.dtype), None
    y = x.float()
    r = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    n = y * r
    dg = (dn * n).sum((0, 1))
    dn = dn * gamma.float()
    return ((dn - n * (dn * n).mean(-1, keepdim=True)) * r).to(x.dtype), dg


def _plain_put(s):
    cos, sin = _cos_sin(s)
    q, k = (_forward(s[n], s[n + "_gamma"], cos, sin, s) for n in "qk")
    at = s["positions"].long()
    live = torch.nonzero(at >= 0)[:, 0]
    at = at[live]
    page = s["table"][live, at // s["page"]].long()
    s["k_cache"][page, :, at % s["page"]] = k[live]
    s["v_cache"][page, :, at % s["page"]] = s["v"][live]
    return q, s["k_cache"], s["v_cache"]


def _plain_attend(s):
    b, n = s["table"].shape
    hq, hk, d = s["q_heads"], s["k_heads"], s["dim"]
    ids = s["table"].clamp(min=0).long()
    # every sequence's keys and values up to the longest: [sequences, heads, tokens, dim]
    k, v = (c[ids].permute(0, 2, 1, 3, 4).reshape(b, hk, -1, d).float() for c in (s["k_cache"], s["v_cache"]))
    live = torch.arange(n * s["page"], device="cuda")[None] < s["lengths"][:, None]
    live &= (s["table"] >= 0).repeat_interleave(s["page"], 1)
    live = live[:, None, None]
    q = s["q"].float().reshape(b, hk, hq // hk, d) * s["scale"]
    score = torch.where(live, torch.matmul(q, k.transpose(2, 3)), -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(live.transpose(2, 3), v, 0.0)) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).reshape(b, hq)
    return o.reshape(b, hq, d).to(s["q"].dtype), lse


def _plain_copy(s):
    src, dst = (torch.from_numpy(s[n].astype(np.int64)).cuda() for n in ("src", "dst"))
    rows = torch.from_numpy(s["rows"]).cuda()
    c = s["cache"]
    live = (torch.arange(s["page"], device="cuda")[None] < rows[:, None])[:, None, :, None]
    c[:, :, dst] = torch.where(live, c[:, :, src], c[:, :, dst])
    return c


def _share(weight, parts):
    """floor(weight parts / 2^24) of whole numbers, weight below 2^62 and parts up to 2^24."""
    return (weight >> 24) * parts + (((weight & 0xFFFFFF) * parts) >> 24)


def _plain_draw(s):
    x = s["logits"].float()
    n, v = x.shape
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    scaled = (x.double() - x[:, :1].double()) * (1.0 / s["temperature"].double())[:, None]
    w = torch.round(torch.exp(scaled) * ONE).long()
    rank = torch.arange(v, device="cuda")[None]
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"], v)[:, None]
        w = torch.where(rank < k, w, 0)
    if s["top_p"] is not None:
        parts = torch.round(s["top_p"].double() * 2 ** 24).long()
        need = _share(w.sum(1), parts)[:, None]
        w = torch.where((torch.cumsum(w, 1) - w < need) | (rank == 0), w, 0)
    if s["min_p"] is not None:
        w = torch.where(w >= torch.round(s["min_p"].double() * ONE).long()[:, None], w, 0)
    w = torch.zeros_like(w).scatter_(1, order, w)  # back in the vocabulary's order
    upto = torch.cumsum(w, 1)
    total = upto[:, -1]
    at = _share(total, (s["u"].double() * 2 ** 24).long())
    token = torch.searchsorted(upto, at[:, None], right=True)
    logprob = torch.log(torch.gather(w, 1, token)[:, 0].double() / total.double())
    return token[:, 0].int(), logprob.float()


def _plain(s):
    if s["op"] == "rotate":
        cos, sin = _cos_sin(s)
        return _forward(s["q"], s["q_gamma"], cos, sin, s), _forward(s["k"], s["k_gamma"], cos, sin, s)
    if s["op"] == "rotate_back":
        cos, sin = _cos_sin(s)
        dq, dq_gamma = _backward(s["dq_out"], s["q"], s["q_gamma"], cos, sin, s)
        dk, dk_gamma = _backward(s["dk_out"], s["k"], s["k_gamma"], cos, sin, s)
        return (dq, dk) if dq_gamma is None else (dq, dk, dq_gamma, dk_gamma)
    return {"rotate_put": _plain_put, "attend": _plain_attend, "copy": _plain_copy, "draw": _plain_draw}[s["op"]](s)


# ---- the library's calls

def _own(s):
    import paper_2609_38095_amd as zo
    if s["op"] == "rotate":
        return zo.zo_norm_rotate(s["q"], s["k"], s["positions"], s["turns"], interleaved=s["interleaved"],
                                 q_gamma=s["q_gamma"], k_gamma=s["k_gamma"], norm_eps=EPS)
    if s["op"] == "rotate_back":
        got = zo.zo_norm_rotate_back(s["dq_out"], s["dk_out"], s["q"], s["k"], s["positions"], s["turns"],
                                     interleaved=s["interleaved"], q_gamma=s["q_gamma"], k_gamma=s["k_gamma"], norm_eps=EPS)
        return got[:2] if s["q_gamma"] is None else got
    if s["op"] == "rotate_put":
        q = zo.zo_norm_rotate_put(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["positions"], s["turns"],
                                  interleaved=s["interleaved"], q_gamma=s["q_gamma"], k_gamma=s["k_gamma"], norm_eps=EPS)
        return q, s["k_cache"], s["v_cache"]
    if s["op"] == "attend":
        return zo.zo_cache_attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["scale"], lse=True)
    if s["op"] == "copy":
        zo.zo_cache_copy(s["k_caches"], s["v_caches"], s["src"], s["dst"], s["rows"])
        return s["cache"]
    return zo.zo_draw(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                      min_p=s["min_p"], logprobs=True)


def run(state):
    return _own(state) if own else _plain(state)


# ---- the least work, and the definitions in 64 bits

def work(case):
    size, d = SIZE[case["dtype"]], case.get("dim", 0)
    if case["op"] in ("rotate", "rotate_back"):
        n = case["tokens"] * (case["q_heads"] + case["k_heads"]) * d
        back = case["op"] == "rotate_back"
        passes = (3 if case["norm"] else 2) if back else 2
        return {"bytes": n * size * passes + 4 * case["tokens"], "flops": n * ((10 if back else 4) * case["norm"] + 3)}
    if case["op"] == "rotate_put":
        n = case["seqs"] * (case["q_heads"] + 2 * case["k_heads"]) * d
        return {"bytes": 2 * n * size + 8 * case["seqs"], "flops": n * (4 * case["norm"] + 3)}
    if case["op"] == "attend":
        # the lengths differ from seed to seed: their mean, the longest among them
        tokens = case["longest"] + (case["seqs"] - 1) * case["longest"] * 2 / 3
        tokens *= 1 - case["empty"]
        q = case["seqs"] * case["q_heads"] * d
        return {"bytes": tokens * case["k_heads"] * d * 2 * size + 2 * q * size + 4 * tokens / case["page"],
                "flops": 4 * tokens * case["q_heads"] * d}
    if case["op"] == "copy":
        rows = case["pairs"] * (case["page"] if case["full"] else (case["page"] + 1) / 2)
        return {"bytes": 2 * 2 * case["layers"] * rows * case["k_heads"] * d * size, "flops": 0}
    return {"bytes": case["seqs"] * case["vocab"] * size, "flops": 4 * case["seqs"] * case["vocab"]}


def _exact_turn(case, x, s):
    """The definition with complex numbers: a pair is one of them, a position a factor of modulus one."""
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


def _exact_rows(case, x, gamma, s):
    if gamma is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS) * gamma
    return _exact_turn(case, x, s)


def _exact_attend(case, s):
    outs, lses = [], []
    for i, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            outs.append(torch.zeros(case["q_heads"], case["dim"], dtype=torch.float64, device="cuda"))
            lses.append(torch.full((case["q_heads"],), -math.inf, dtype=torch.float64, device="cuda"))
            continue
        pages = s["table"][i, :-(-n // case["page"])].long()
        k, v = (c[pages].transpose(0, 1).reshape(case["k_heads"], -1, case["dim"])[:, :n].double()
                for c in (s["k_cache"], s["v_cache"]))
        q = s["q"][i].double().reshape(case["k_heads"], -1, case["dim"])
        score = torch.matmul(k, (q * s["scale"]).transpose(1, 2).contiguous())  # [heads, tokens, group]
        lse = torch.logsumexp(score, 1)
        out = torch.matmul(torch.exp(score - lse[:, None]).transpose(1, 2).contiguous(), v)
        outs.append(out.reshape(case["q_heads"], case["dim"]))
        lses.append(lse.reshape(-1))
    return torch.stack(outs), torch.stack(lses)


def _exact_draw(case, s):
    tokens, logprobs = [], []
    for i in range(case["seqs"]):
        x = s["logits"][i].double().cpu().numpy()
        w = np.exp((x - x.max()) / float(s["temperature"][i]))
        order = np.argsort(-x, kind="stable")
        keep = len(x)
        if s["top_k"] is not None and int(s["top_k"][i]) > 0:
            keep = min(keep, int(s["top_k"][i]))
        if s["top_p"] is not None:
            sums = np.cumsum(w[order[:keep]])
            keep = min(keep, 1 + int(np.searchsorted(sums, float(s["top_p"][i]) * sums[-1])))
        kept = order[:keep]
        if s["min_p"] is not None:
            kept = kept[w[kept] >= float(s["min_p"][i])]
        kept = np.sort(kept)
        sums = np.cumsum(w[kept])
        u = math.floor(float(s["u"][i]) * 2 ** 24) / 2 ** 24
        j = min(int(np.searchsorted(sums, u * sums[-1], side="right")), len(kept) - 1)
        tokens.append(int(kept[j]))
        logprobs.append(math.log(w[kept[j]] / sums[-1]))
    return np.array(tokens, np.int32), np.array(logprobs)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rotate", "rotate_back", "rotate_put"):
        names = ("q", "k")
        x = [s[n].double().requires_grad_() for n in names]
        gamma = [s[n + "_gamma"].double().requires_grad_() if case["norm"] else None for n in names]
        y = [_exact_rows(case, a, b, s) for a, b in zip(x, gamma)]
        if case["op"] == "rotate":
            return tuple(t.detach() for t in y)
        if case["op"] == "rotate_back":
            grads = torch.autograd.grad(y, x + (gamma if case["norm"] else []), [s["dq_out"].double(), s["dk_out"].double()])
            return tuple(grads)
        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        for i, at in enumerate(s["positions"].tolist()):
            if at >= 0:
                page = int(s["table"][i, at // case["page"]])
                k_cache[page, :, at % case["page"]] = y[1][i].detach()
                v_cache[page, :, at % case["page"]] = s["v"][i].double()
        return y[0].detach(), k_cache, v_cache
    if case["op"] == "attend":
        return _exact_attend(case, s)
    if case["op"] == "copy":
        return None  # nothing is computed
    return _exact_draw(case, s)
