"""SPSA on a score that has no gradient: a reward of the answers that a model writes.

A small OPT-shaped decoder (random weights) is perturbed with theta +- eps z; under each perturbation it writes
several answers to each prompt and their reward is the score. The projected gradient becomes one byte, and the
byte is applied as any machine would apply it. Both evaluations draw their tokens with the same random words, so
that the two rewards differ by the weights alone.

    python examples/spsa_answers.py --steps 5

What is used of the library, in the order of an evaluation: jb_perturb, jb_cache_reserve (pages for the prompts),
jb_cache_write and jb_attend (the prompts' tokens as queries of their rows), jb_cache_fork (several answers to one
prompt), then for each token jb_cache_reserve, jb_cache_write, jb_attend and jb_sample; jb_cache_free and
jb_cache_compact when half of an answer's length is written and some have ended, jb_cache_free at the end;
jb_quantize_grad and jb_apply_updates.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2306_10015_gb300 as jb  # noqa: E402

END = 2  # the token that ends an answer


class Decoder:
    """OPT's layout: learned positions, layer norm before attention and before the ReLU network, tied head."""

    def __init__(self, layers=2, d=256, heads=4, ffn=1024, vocab=512, positions=128, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.layers, self.d, self.heads, self.vocab, self.dtype = layers, d, heads, vocab, dtype
        w = lambda *shape: (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).to(dtype)  # noqa: E731
        self.p = {"tokens": w(vocab, d), "positions": w(positions, d), "norm": torch.ones(d, device="cuda", dtype=dtype)}
        for i in range(layers):
            self.p.update({f"{i}.qkv": w(3 * d, d), f"{i}.out": w(d, d), f"{i}.fc1": w(ffn, d), f"{i}.fc2": w(d, ffn),
                           f"{i}.norm1": torch.ones(d, device="cuda", dtype=dtype), f"{i}.norm2": torch.ones(d, device="cuda", dtype=dtype)})
        self.table = jb.ParamTable(self.p.values())

    def cache(self, rows, tokens, page=16):
        """A cache with room for `rows` rows of `tokens` tokens."""
        row_pages = -(-tokens // page)
        pages = jb.PageTable.empty(rows, row_pages, rows * row_pages, page)
        shape = (rows * row_pages, self.heads, page, self.d // self.heads)
        new = lambda: [torch.empty(shape, dtype=self.dtype, device="cuda") for _ in range(self.layers)]  # noqa: E731
        return jb.KVCache(pages, new(), new())

    def logits(self, cache, tokens, rows, pos):
        """Logits after each of the tokens: token i is written to position pos[i] of row rows[i] (pos -1: nothing)."""
        p, n = self.p, tokens.shape[0]
        x = p["tokens"][tokens.long()] + p["positions"][pos.clamp(min=0).long()]
        norm = lambda v, w: F.layer_norm(v.float(), (self.d,)).to(self.dtype) * w  # noqa: E731
        for i in range(self.layers):
            q, k, v = (norm(x, p[f"{i}.norm1"]) @ p[f"{i}.qkv"].T).view(n, 3 * self.heads, -1).split(self.heads, 1)
            jb.jb_cache_write(cache, i, k, v, rows, pos)
            o = jb.jb_attend(cache, i, q, rows, pos)
            x = x + o.view(n, self.d) @ p[f"{i}.out"].T
            x = x + F.relu(norm(x, p[f"{i}.norm2"]) @ p[f"{i}.fc1"].T) @ p[f"{i}.fc2"].T
        return norm(x, p["norm"]) @ p["tokens"].T


def random_words(seed, n):
    """n 32-bit words of the seed's own stream, far from the blocks that perturb weights."""
    out = torch.empty(4 * -(-n // 4), dtype=torch.int32, device="cuda")
    jb.jb_debug_philox(seed, 1 << 60, out.shape[0] // 4, out)
    return out[:n]


def write_answers(model, prompts, answers, length, seed, temperature=1.0, top_p=0.95):
    """`answers` answers of up to `length` tokens to each prompt ([n, t] int32): tokens [n * answers, length],
    -1 after an answer's end, and their log-probabilities."""
    n, t = prompts.shape
    rows = n * answers
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = model.cache(n + rows, t + length + 16)
    every = torch.arange(n + rows, **i32)
    prompt_rows, answer_rows = every[:n], every[n:]

    # the prompts, all their tokens at once but the last one, which the answers start from
    jb.jb_cache_reserve(cache, prompt_rows, torch.full((n,), t - 1, **i32))
    at = torch.arange(t - 1, **i32).repeat(n)
    model.logits(cache, prompts[:, :-1].reshape(-1), prompt_rows.repeat_interleave(t - 1), at)
    jb.jb_cache_fork(cache, prompt_rows.repeat_interleave(answers), answer_rows)
    jb.jb_cache_free(cache, prompt_rows)

    words = random_words(seed, rows * length).view(length, rows)
    tokens = prompts[:, -1].repeat_interleave(answers).contiguous()
    alive = torch.ones(rows, dtype=torch.bool, device="cuda")
    out, logprobs = torch.full((length, rows), -1, **i32), torch.zeros(length, rows, device="cuda")
    for step in range(length):
        if step == length // 2:  # rows that have ended give their pages back
            jb.jb_cache_free(cache, torch.where(alive, -1, answer_rows))
            jb.jb_cache_compact(cache)
        pos = torch.where(alive, cache.pages.lens[n:], -1)
        jb.jb_cache_reserve(cache, answer_rows, alive.int())
        logits = model.logits(cache, tokens, answer_rows, pos)
        tokens, lp = jb.jb_sample(logits, words[step], temperature=temperature, top_p=top_p)
        out[step] = torch.where(alive, tokens, -1)
        logprobs[step] = torch.where(alive, lp, 0.0)
        alive = alive & (tokens != END)
    jb.jb_cache_free(cache, answer_rows)
    return out.T, logprobs.T


def reward(answers, vocab):
    """The share of an answer's tokens in the lower half of the vocabulary: no gradient to be had."""
    real = answers >= 0
    return ((answers < vocab // 2) & real).sum().item() / max(1, real.sum().item())


def train(steps=5, prompts=4, answers=8, length=24, eps=2e-2, lr=2e-3, qscale=16.0, seed=0, log=print):
    """The rewards (theta + eps z, theta - eps z) and byte of each step, and the model."""
    model = Decoder(seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    asked = torch.randint(3, model.vocab, (prompts, 9), generator=g, device="cuda", dtype=torch.int32)
    machine, history = 1_700_000_000_000_000_000 + seed, []
    for step in range(steps):
        s = (machine, step, 0)
        jb.jb_perturb(model.table, s, eps)
        plus = reward(write_answers(model, asked, answers, length, s)[0], model.vocab)
        jb.jb_perturb(model.table, s, -2 * eps)
        minus = reward(write_answers(model, asked, answers, length, s)[0], model.vocab)
        jb.jb_perturb(model.table, s, eps)
        # the update descends, and a reward is to grow
        byte = jb.jb_quantize_grad(-(plus - minus) / (2 * eps), qscale)
        jb.jb_apply_updates(model.table, [s], [byte], lr, denom=1.0, qscale=qscale)
        history.append((plus, minus, byte))
        log(f"step {step}: reward {plus:.4f} / {minus:.4f}, byte {byte}")
    return history, model


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description="SPSA on a reward of written answers")
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    train(steps=a.steps, seed=a.seed)
