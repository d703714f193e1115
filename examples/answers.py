"""1.5-SPSA on a score of sampled answers.

A zero-order step needs one number for each probe and nothing of how it came about, so it can train on
what a model answers. Here a small Qwen3-shaped decoder (random weights, one flat buffer) answers a few
prompts several times each, and the loss is the share of drawn tokens outside a wanted set. Per probe
the weights are perturbed in place, the answers are drawn again with the same random numbers, and the
step is the usual one: coefficients from the losses, one fused update.

    python examples/answers.py [--steps N] [--probes K] [--answers A] [--tokens T] [--temperature X] [--eps E] [--drafted]

The answers take the operators of a decode step: each prompt's keys and values are put in the paged cache once, its
tokens attending together as a chain, and its pages are shared by all answers to it (a page is copied when the first answer
writes into it); each new token's queries and keys are normed, rotated and put in one pass, attend to the cache, and the
next token is drawn from the logits.

With --drafted the clean answers are drafts of a probe's: the model reads several drafted tokens of every answer at once,
draws behind each of them, and keeps the longest beginning that the draws agree with. The answers are the same ones up to
rounding: in bf16 a draw among many tokens of nearly equal weight can be another one, and the answer goes on from there (at the defaults 204
of 512 answers drafted by themselves; none at --temperature 0, none in fp32). How many passes that saves is a matter of how alike the probes are: of 11, an
answer takes 3.0 at --temperature 0 --eps 1e-5 and 7.5 at --eps 1e-3, but all 11 at the defaults, where these random weights
have no favourite token and eps is as large as they are.
"""

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2609_38095_amd as zo  # noqa: E402
import workloads  # noqa: E402

SMALL = workloads.Workload("answers", "bf16", (8,), 2e-2, 2e-2, hidden=256, layers=2, ffn=512, family="qwen3",
                           heads=8, kv_heads=4, tied=True)
EPS = 1e-6
ROTARY_BASE = 1e6
PAGE = 16


def rms_norm(x, gamma):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)).to(x.dtype) * gamma


class Decoder:
    """A Qwen3-shaped decoder whose weights are views of one flat buffer, with a paged cache for each layer."""

    def __init__(self, w, theta, pages):
        self.w, self.dim = w, workloads.QWEN3_HEAD_DIM
        self.at = {name: theta[o:o + n] for name, o, n in workloads.tensor_offsets(w)}
        starts = {name: o for name, o, _ in workloads.tensor_offsets(w)}
        h, hq, hk = w.hidden, w.heads * self.dim, w.kv_heads * self.dim
        # the three projections lie one after another: one product
        self.qkv = [theta[starts[f"layers.{i}.q_proj.weight"]:][:(hq + 2 * hk) * h].view(-1, h) for i in range(w.layers)]
        self.up = [theta[starts[f"layers.{i}.gate_proj.weight"]:][:2 * w.ffn * h].view(-1, h) for i in range(w.layers)]
        shape = (w.layers, 2, pages, w.kv_heads, PAGE, self.dim)
        self.cache = torch.zeros(shape, dtype=theta.dtype, device=theta.device)
        self.turns = zo.zo_rotary_turns(self.dim, ROTARY_BASE)

    def caches(self):
        return [c[0] for c in self.cache], [c[1] for c in self.cache]

    def _behind(self, tokens, attention):
        """Logits behind tokens whose attention (layer, queries, keys and values as rows of heads) is given."""
        w, at = self.w, self.at
        x = at["embed_tokens"].view(-1, w.hidden)[tokens.long()]
        for i in range(w.layers):
            p = f"layers.{i}."
            qkv = (rms_norm(x, at[p + "input_norm.gamma"]) @ self.qkv[i].T).view(len(tokens), -1, self.dim)
            o = attention(i, *qkv.split((w.heads, w.kv_heads, w.kv_heads), dim=1))
            x = x + o.flatten(1) @ at[p + "o_proj.weight"].view(w.hidden, -1).T
            gate, up = (rms_norm(x, at[p + "post_attn_norm.gamma"]) @ self.up[i].T).chunk(2, dim=1)
            x = x + (torch.nn.functional.silu(gate) * up) @ at[p + "down_proj.weight"].view(w.hidden, -1).T
        return rms_norm(x, at["final_norm.gamma"]) @ at["embed_tokens"].view(-1, w.hidden).T

    def _put(self, i, q, k, v, table, positions, **places):
        gamma = {n + "_gamma": self.at[f"layers.{i}.{n}_norm.gamma"] for n in "qk"}
        return zo.zo_norm_rotate_put(q, k, v, *self.cache[i], table, positions, self.turns, norm_eps=EPS, **gamma, **places)

    def logits(self, tokens, table, positions):
        """Logits behind one new token of each sequence (a row of the table) at its position, whose keys and values go into the cache."""
        lengths = positions + 1

        def attention(i, q, k, v):
            return zo.zo_cache_attend(self._put(i, q, k, v, table, positions), *self.cache[i], table, lengths)
        return self._behind(tokens, attention)

    def tree_logits(self, tokens, table, starts, lengths, parents=None, words=1):
        """Logits behind several new tokens of each sequence, whose keys and values go into the cache behind its lengths[s]: a chain
        (a prompt), or the tree that parents makes of them."""
        seqs, positions, places, seen = zo.zo_tree_lay(starts, lengths, len(tokens), parents, words if parents is not None else 0)

        def attention(i, q, k, v):
            q = self._put(i, q, k, v, table, positions, seqs=seqs, places=places)
            return zo.zo_tree_attend(q, *self.cache[i], table, lengths, starts, seen)
        return self._behind(tokens, attention)


def _settings(n, dev, temperature, top_k, top_p):
    return dict(temperature=torch.full((n,), temperature, device=dev), top_k=torch.full((n,), top_k, dtype=torch.int32, device=dev),
                top_p=torch.full((n,), top_p, device=dev), logprobs=True)


def _on(dev, a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev)


def _starts(counts):
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int32)


def _read_prompts(model, prompts, answers):
    """(book, sequences of `answers` answers to each prompt, logits behind each prompt): all prompts in one pass."""
    dev = model.cache.device
    book = zo.ZoPages(model.cache.shape[2], PAGE)
    prompt_seqs = [book.add(len(p)) for p in prompts]
    ids, lengths = book.table(prompt_seqs)
    starts = _starts(lengths)
    logits = model.tree_logits(_on(dev, np.concatenate(prompts)), _on(dev, ids), _on(dev, starts), torch.zeros(len(prompts), dtype=torch.int32, device=dev))
    # the answers share the prompt's pages and begin with a draw from the logits behind it
    held = [book.fork(s) for s in prompt_seqs for _ in range(answers)]
    for s in prompt_seqs:
        book.drop(s)
    return book, held, logits[_on(dev, np.repeat(starts[1:] - 1, answers))]


def _extend(model, book, held, counts):
    """Room for counts[i] more tokens of sequence held[i], each in pages of its own."""
    moves = [m for m in (book.extend(s, n) for s, n in zip(held, counts)) if m is not None]
    if moves:
        zo.zo_cache_copy(*model.caches(), *zip(*moves))


def answer(model, prompts, answers, u, temperature=1.0, top_k=200, top_p=0.95):
    """Tokens and log probabilities [prompts * answers, steps] of `answers` answers to each prompt, drawn with
    the random numbers u [steps, prompts * answers]."""
    dev = model.cache.device
    book, held, logits = _read_prompts(model, prompts, answers)
    n, steps = len(held), u.shape[0]
    settings = _settings(n, dev, temperature, top_k, top_p)
    tokens, logprobs = [], []
    for step in range(steps):
        drawn, lp = zo.zo_draw(logits, u[step], **settings)
        tokens.append(drawn)
        logprobs.append(lp)
        if step + 1 == steps:
            break
        _extend(model, book, held, [1] * n)
        ids, lengths = book.table(held)
        logits = model.logits(drawn, _on(dev, ids), _on(dev, lengths - 1))
    return torch.stack(tokens, 1), torch.stack(logprobs, 1)


def _tree(token, drafts):
    """(tokens, parents, depths) of a tree: `token`, and behind it the drafts, whose common beginnings are shared."""
    tokens, parents, depths, after = [token], [-1], [0], {}
    for draft in drafts:
        at = 0
        for t in draft:
            if (at, t) not in after:
                after[at, t] = len(tokens)
                tokens.append(t)
                parents.append(at)
                depths.append(depths[at] + 1)
            at = after[at, t]
    return tokens, parents, depths


def answer_drafted(model, prompts, answers, u, drafts, ahead=4, temperature=1.0, top_k=200, top_p=0.95):
    """(tokens, log probabilities, passes of each answer): the answers of answer() by way of drafts, a list of earlier answers' tokens [prompts * answers, any]
    each. In each pass the model reads up to `ahead` tokens of every draft of an answer that has its last token at the same place."""
    dev = model.cache.device
    drafts = [d.cpu().tolist() for d in drafts]
    book, held, logits = _read_prompts(model, prompts, answers)
    n, steps = len(held), u.shape[0]
    first, lp = zo.zo_draw(logits, u[0], **_settings(n, dev, temperature, top_k, top_p))
    tokens, logprobs, passes = [[t] for t in first.tolist()], [[x] for x in lp.tolist()], [0] * n
    while True:
        live = [i for i in range(n) if len(tokens[i]) < steps]
        if not live:
            break
        trees = []
        for i in live:
            have = len(tokens[i])
            behind = [d[i][have:min(have + ahead, steps - 1)] for d in drafts if d[i][have - 1:have] == tokens[i][-1:]]
            trees.append(_tree(tokens[i][-1], behind))
        counts = [len(t[0]) for t in trees]
        lengths = np.array([book.length(held[i]) for i in live], np.int32)
        _extend(model, book, [held[i] for i in live], counts)
        table = _on(dev, book.table([held[i] for i in live])[0])
        drafted, parents = (_on(dev, np.concatenate([np.array(t[k], np.int32) for t in trees])) for k in (0, 1))
        starts, dev_lengths = _on(dev, _starts(counts)), _on(dev, lengths)
        words = -(-max(counts) // 64)
        logits = model.tree_logits(drafted, table, starts, dev_lengths, parents, words)
        # the token behind each is drawn with the random number of its place in its answer
        at = np.concatenate([len(tokens[i]) + np.array(t[2]) for i, t in zip(live, trees)])
        drawn, lp = zo.zo_draw(logits, u[_on(dev, at), _on(dev, np.repeat(live, counts))], **_settings(len(at), dev, temperature, top_k, top_p))
        path, won, walked = zo.zo_tree_accept(drafted, drawn, starts, ahead + 1, parents, words=words)
        zo.zo_tree_keep(*model.caches(), table, dev_lengths, path)
        rows = torch.gather(lp[(starts[:-1, None] + path.clamp(min=0)).long()], 1, torch.arange(ahead + 1, device=dev)[None].expand_as(path))
        won, walked, rows = won.tolist(), walked.tolist(), rows.tolist()
        for k, i in enumerate(live):
            tokens[i] += won[k][:walked[k]]
            logprobs[i] += rows[k][:walked[k]]
            book.cut(held[i], int(lengths[k]) + walked[k])
            passes[i] += 1
    return torch.tensor(tokens, dtype=torch.int32, device=dev), torch.tensor(logprobs, device=dev), passes


def pages_needed(prompts, answers, steps):
    """Room for every answer's own copy of its last prompt page and what it adds (a draft of up to a page too), and the prompts."""
    return sum(-(-len(p) // PAGE) + answers * (3 + steps // PAGE) for p in prompts)


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=5)
    parser.add_argument("--probes", type=int, default=SMALL.K[0])
    parser.add_argument("--answers", type=int, default=16)
    parser.add_argument("--tokens", type=int, default=12)
    parser.add_argument("--temperature", type=float, default=1.0)
    parser.add_argument("--eps", type=float, default=SMALL.eps)
    parser.add_argument("--drafted", action="store_true", help="draft each probe's answers by the clean ones")
    args = parser.parse_args()
    w, dev = SMALL, torch.device("cuda")
    theta = torch.empty(w.n, dtype=torch.bfloat16, device=dev)
    workloads.fill_model_buffer_device(theta, w)
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, workloads.QWEN3_VOCAB, n).astype(np.int32) for n in (5, 21, 38)]
    model = Decoder(w, theta, pages_needed(prompts, args.answers, args.tokens))
    g = torch.Generator(device=dev)

    drafts, passes = [], []

    def loss(step, probe=True):
        """The share of drawn tokens that are odd; the same random numbers for every probe of a step."""
        g.manual_seed(step)
        u = torch.rand(args.tokens, len(prompts) * args.answers, generator=g, device=dev)
        if probe and args.drafted:
            tokens, _, count = answer_drafted(model, prompts, args.answers, u, drafts, temperature=args.temperature)
            passes.extend(count)
        else:
            tokens, _ = answer(model, prompts, args.answers, u, args.temperature)
            drafts[:] = [tokens]
        return float((tokens % 2).double().mean())

    for step in range(args.steps):
        seed, K = 0, args.probes
        clean, plus, minus = loss(step, probe=False), np.zeros(K), np.zeros(K)
        for k in range(K):
            zo.zo_perturb(theta, k, args.eps, seed, step)
            plus[k] = loss(step)
            zo.zo_perturb(theta, k, -2 * args.eps, seed, step)
            minus[k] = loss(step)
            zo.zo_perturb(theta, k, args.eps, seed, step)
        zo.zo_update(theta, zo.zo_probe_coeffs(plus, minus, clean, args.eps), w.lr, seed, step)
        read = f", {np.mean(passes):.1f} passes an answer for {args.tokens - 1}" if passes else ""
        print(f"step {step}: odd tokens {clean:.4f}, probes {plus.mean():.4f} / {minus.mean():.4f}{read}", flush=True)


if __name__ == "__main__":
    main()
