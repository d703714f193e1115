"""1.5-SPSA on a score of sampled answers.

A zero-order step needs one number for each probe and nothing of how it came about, so it can train on
what a model answers. Here a small Qwen3-shaped decoder (random weights, one flat buffer) answers a few
prompts several times each, and the loss is the share of drawn tokens outside a wanted set. Per probe
the weights are perturbed in place, the answers are drawn again with the same random numbers, and the
step is the usual one: coefficients from the losses, one fused update.

    python examples/answers.py [--steps N] [--probes K] [--answers A] [--tokens T]

The answers take the operators of a decode step: the prompt's keys and values are put in the paged
cache once and its pages shared by all answers to it (a page is copied when the first answer writes
into it), each new token's queries and keys are normed, rotated and put in one pass, attend to the
cache, and the next token is drawn from the logits. A prompt's tokens attend one by one, as sequences
that share their pages: right for prompts of this size, but each token reads what is before it again.
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

    def logits(self, tokens, table, positions, seqs=None):
        """Logits behind tokens at their positions of their sequences (row t of the table for token t, or row seqs[t]),
        whose keys and values go into the cache. Each token attends to its sequence up to itself, so a prompt's
        tokens can be given at once."""
        w, at = self.w, self.at
        rows = table if seqs is None else table[seqs.long()]
        lengths = positions + 1
        x = at["embed_tokens"].view(-1, w.hidden)[tokens.long()]
        for i in range(w.layers):
            p = f"layers.{i}."
            qkv = (rms_norm(x, at[p + "input_norm.gamma"]) @ self.qkv[i].T).view(len(tokens), -1, self.dim)
            q, k, v = qkv.split((w.heads, w.kv_heads, w.kv_heads), dim=1)
            k_cache, v_cache = self.cache[i]
            q = zo.zo_norm_rotate_put(q, k, v, k_cache, v_cache, table, positions, self.turns, q_gamma=at[p + "q_norm.gamma"],
                                      k_gamma=at[p + "k_norm.gamma"], norm_eps=EPS, seqs=seqs)
            o = zo.zo_cache_attend(q, k_cache, v_cache, rows, lengths)
            x = x + o.flatten(1) @ at[p + "o_proj.weight"].view(w.hidden, -1).T
            gate, up = (rms_norm(x, at[p + "post_attn_norm.gamma"]) @ self.up[i].T).chunk(2, dim=1)
            x = x + (torch.nn.functional.silu(gate) * up) @ at[p + "down_proj.weight"].view(w.hidden, -1).T
        return rms_norm(x, at["final_norm.gamma"]) @ at["embed_tokens"].view(-1, w.hidden).T


def answer(model, prompts, answers, u, temperature=1.0, top_k=200, top_p=0.95):
    """Tokens and log probabilities [prompts * answers, steps] of `answers` answers to each prompt, drawn with
    the random numbers u [steps, prompts * answers]."""
    dev = model.cache.device
    book = zo.ZoPages(model.cache.shape[2], PAGE)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
    # every token of every prompt but its last, in one pass
    prompt_seqs = [book.add(len(p)) for p in prompts]
    ids, lengths = book.table(prompt_seqs)
    seqs = np.repeat(np.arange(len(prompts), dtype=np.int32), lengths)
    positions = np.concatenate([np.arange(n, dtype=np.int32) for n in lengths])
    logits = model.logits(put(np.concatenate(prompts)), put(ids), put(positions), put(seqs))
    # the answers share the prompt's pages and begin with a draw from the logits behind it
    held = [book.fork(s) for s in prompt_seqs for _ in range(answers)]
    for s in prompt_seqs:
        book.drop(s)
    logits = logits[put(np.repeat(np.cumsum(lengths) - 1, answers))]
    n, steps = len(held), u.shape[0]
    settings = dict(temperature=torch.full((n,), temperature, device=dev), top_k=torch.full((n,), top_k, dtype=torch.int32, device=dev),
                    top_p=torch.full((n,), top_p, device=dev), logprobs=True)
    tokens, logprobs = [], []
    for step in range(steps):
        drawn, lp = zo.zo_draw(logits, u[step], **settings)
        tokens.append(drawn)
        logprobs.append(lp)
        if step + 1 == steps:
            break
        moves = [m for m in (book.extend(s) for s in held) if m is not None]
        if moves:
            zo.zo_cache_copy(*model.caches(), *zip(*moves))
        ids, lengths = book.table(held)
        logits = model.logits(drawn, put(ids), put(lengths - 1))
    return torch.stack(tokens, 1), torch.stack(logprobs, 1)


def pages_needed(prompts, answers, steps):
    """Room for every answer's own copy of its last prompt page and what it adds, and the prompts."""
    return sum(-(-len(p) // PAGE) + answers * (2 + steps // PAGE) for p in prompts)


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=5)
    parser.add_argument("--probes", type=int, default=SMALL.K[0])
    parser.add_argument("--answers", type=int, default=16)
    parser.add_argument("--tokens", type=int, default=12)
    args = parser.parse_args()
    w, dev = SMALL, torch.device("cuda")
    theta = torch.empty(w.n, dtype=torch.bfloat16, device=dev)
    workloads.fill_model_buffer_device(theta, w)
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, workloads.QWEN3_VOCAB, n).astype(np.int32) for n in (5, 21, 38)]
    model = Decoder(w, theta, pages_needed(prompts, args.answers, args.tokens))
    g = torch.Generator(device=dev)

    def loss(step):
        """The share of drawn tokens that are odd; the same random numbers for every probe of a step."""
        g.manual_seed(step)
        u = torch.rand(args.tokens, len(prompts) * args.answers, generator=g, device=dev)
        tokens, _ = answer(model, prompts, args.answers, u)
        return float((tokens % 2).double().mean())

    for step in range(args.steps):
        seed, K = 0, args.probes
        clean, plus, minus = loss(step), np.zeros(K), np.zeros(K)
        for k in range(K):
            zo.zo_perturb(theta, k, w.eps, seed, step)
            plus[k] = loss(step)
            zo.zo_perturb(theta, k, -2 * w.eps, seed, step)
            minus[k] = loss(step)
            zo.zo_perturb(theta, k, w.eps, seed, step)
        zo.zo_update(theta, zo.zo_probe_coeffs(plus, minus, clean, w.eps), w.lr, seed, step)
        print(f"step {step}: odd tokens {clean:.4f}, probes {plus.mean():.4f} / {minus.mean():.4f}", flush=True)


if __name__ == "__main__":
    main()
