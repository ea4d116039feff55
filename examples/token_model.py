"""A small token model with a LAPLEX^(r) vocabulary head, through the library's entry points: embedding, rotary positions,
attention with a decay for each head, the head, log probabilities.  Trains on a synthetic text, reads a prompt, and writes on
from it token by token.

    python examples/token_model.py [--vocabulary 500] [--width 128] [--heads 4] [--steps 60] [--dtype bf16]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

from paper_2605_24584_amd import binding as B


class Workspaces:
    """One workspace per kind of call, grown when a larger call comes."""

    def __init__(self):
        self.kept = {}

    def __call__(self, name, size):
        if name not in self.kept or self.kept[name].numel() < size:
            self.kept[name] = torch.empty(size, dtype=torch.uint8, device="cuda")
        return self.kept[name]


class TokenModel:
    def __init__(self, vocabulary, width, heads, operators=4, dtype=torch.float32, context=4096, stretch=1.0, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        uniform = lambda *s: torch.rand(*s, generator=gen, device="cuda")
        self.vocabulary, self.width, self.heads, self.dim, self.dtype = vocabulary, width, heads, width // heads, dtype
        span = (vocabulary + width) / 64.0
        self.weights = {
            "embedding": normal(vocabulary, width),
            "qkv": normal(width, 3 * width) / math.sqrt(width),
            "out": normal(width, width) / math.sqrt(width),
            # the head: logits = sum_q w[q] L(a[q], b[q]) x
            "a": uniform(operators, vocabulary) * span, "b": uniform(operators, width) * span, "w": normal(operators) / operators,
        }
        # decay lengths from 8 tokens to 1024
        self.rates = torch.exp(-torch.linspace(math.log(8.0), math.log(1024.0), heads, device="cuda"))
        self.frequencies = torch.empty(self.dim // 2, device="cuda")
        B.laplex_rotary_frequencies(self.frequencies, 10000.0, B.LAPLEX_ROTARY_PARTS if stretch > 1.0 else B.LAPLEX_ROTARY_PLAIN, stretch, context)
        self.magnitude = 0.1 * math.log(stretch) + 1.0
        self.scale = 1.0 / math.sqrt(self.dim)
        self.workspace = Workspaces()

    # --- forward ------------------------------------------------------------------------------------------------------

    def _project(self, tokens, positions):
        """Embedded tokens and their queries, keys (turned, in place) and values: parts of one matrix."""
        x = self.weights["embedding"][tokens]
        qkv = (x @ self.weights["qkv"]).to(self.dtype)
        heads = qkv.view(len(tokens), 3 * self.heads, self.dim)
        turned = heads[:, :2 * self.heads]
        B.laplex_rotary(turned, positions, self.frequencies, turned, self.magnitude)
        return x, heads[:, :self.heads], heads[:, self.heads:2 * self.heads], heads[:, 2 * self.heads:]

    def _head(self, x, y, save=False):
        """Logits (vocabulary, tokens) of x + y out."""
        hidden = (x + y.float().reshape(x.shape) @ self.weights["out"]).T.contiguous()
        a, b, w = (self.weights[n] for n in "abw")
        logits = torch.empty(self.vocabulary, hidden.shape[1], device="cuda")
        ws = self.workspace("head", B.laplex_mix_workspace_bytes(len(w), self.vocabulary, self.width, hidden.shape[1]))
        B.laplex_mix_apply(a, b, w, hidden, logits, ws, B.LAPLEX_SAVE_SCANS if save else 0)
        return hidden, logits, ws

    def _logprob(self, logits, targets, top=0):
        t = logits.shape[1]
        new = lambda *s: torch.empty(*s, device="cuda")
        logp, lse, entropy = new(t) if targets is not None else None, new(t), new(t)
        ids, alternatives = (torch.empty(top, t, dtype=torch.int64, device="cuda"), new(top, t)) if top else (None, None)
        B.laplex_logprob(logits, targets, logp, lse, entropy, ids, alternatives,
                         self.workspace("logprob", B.laplex_logprob_workspace_bytes(self.vocabulary, t, top)))
        return logp, lse, entropy, ids, alternatives

    def _attend(self, q, k, v, sequences, starts, state_in, state_out):
        y = torch.empty(v.shape, device="cuda", dtype=self.dtype)
        ws = self.workspace("attention", B.laplex_decay_attention_workspace_bytes(self.dtype, len(q), sequences, self.heads, self.dim, self.dim))
        B.laplex_decay_attention(q, k, v, self.rates, y, ws, self.scale, sequences, starts, state_in, state_out)
        return y, ws

    def new_state(self, sequences):
        return torch.zeros(sequences, self.heads, self.dim, self.dim, device="cuda")

    def read(self, tokens, positions, starts=None, state=None, targets=None, top=0):
        """Reads prompts that lie one behind the other (from row starts[b] on); `state` is carried on in place.
        (log probabilities of the targets, if there are any, entropies, ids and log probabilities of the likeliest tokens)"""
        sequences = 1 if starts is None else len(starts) - 1
        x, q, k, v = self._project(tokens, positions)
        y, _ = self._attend(q, k, v, sequences, starts, state, state)
        _, logits, _ = self._head(x, y)
        logp, _, entropy, ids, alternatives = self._logprob(logits, targets, top)
        return logp, entropy, ids, alternatives

    def write(self, tokens, positions, state, top=1):
        """One more token of every sequence: what comes next, likeliest first, and its log probability."""
        x, q, k, v = self._project(tokens, positions)
        y = torch.empty(v.shape, device="cuda", dtype=self.dtype)
        B.laplex_decay_attention_step(q, k, v, self.rates, state, y, self.scale)
        _, logits, _ = self._head(x, y)
        _, _, entropy, ids, alternatives = self._logprob(logits, None, top)
        return ids, alternatives, entropy

    # --- training -----------------------------------------------------------------------------------------------------

    def gradients(self, tokens, positions, targets, starts=None, entropy_bonus=0.0):
        """(mean of -logp - entropy_bonus * entropy over the tokens that have a target, gradients of all weights)"""
        sequences = 1 if starts is None else len(starts) - 1
        W = self.weights
        x, q, k, v = self._project(tokens, positions)
        y, attention_ws = self._attend(q, k, v, sequences, starts, None, None)
        hidden, logits, head_ws = self._head(x, y, save=True)
        logp, lse, entropy, _, _ = self._logprob(logits, targets)
        given = (targets >= 0) & (targets < self.vocabulary)
        share = given.float() / given.sum().clamp(min=1)
        loss = -((logp + entropy_bonus * entropy) * share).sum()

        # the gradient of the logits takes their place
        B.laplex_logprob_backward(logits, targets, lse, entropy, -share, -entropy_bonus * share, None, logits)
        g = {n: torch.empty_like(W[n]) for n in "abw"}
        ghidden = torch.empty_like(hidden)
        B.laplex_mix_apply_backward(W["a"], W["b"], W["w"], hidden, logits, ghidden, g["a"], g["b"], g["w"], head_ws,
                                    B.LAPLEX_SAVE_SCANS | B.LAPLEX_REUSE_PLAN)
        gx = ghidden.T
        flat = y.float().reshape(x.shape)
        g["out"] = flat.T @ gx
        gy = (gx @ W["out"].T).to(self.dtype).view(y.shape)
        gqkv = torch.empty(len(tokens), 3 * self.heads, self.dim, device="cuda", dtype=self.dtype)
        gq, gk, gv = (gqkv[:, i * self.heads:(i + 1) * self.heads] for i in range(3))
        B.laplex_decay_attention_backward(q, k, v, self.rates, gy, gq, gk, gv, attention_ws, self.scale, sequences, starts)
        turned = gqkv[:, :2 * self.heads]
        B.laplex_rotary(turned, positions, self.frequencies, turned, self.magnitude, B.LAPLEX_ROTARY_INVERSE)
        gqkv = gqkv.float().view(len(tokens), -1)
        g["qkv"] = x.T @ gqkv
        g["embedding"] = torch.zeros_like(W["embedding"]).index_add_(0, tokens, gx + gqkv @ W["qkv"].T)
        return loss, g

    def step(self, gradients, rate):
        for name, g in gradients.items():
            self.weights[name].sub_(g, alpha=rate)


def text(vocabulary, length, seed=1):
    """A synthetic text: a few phrases over and over."""
    gen = torch.Generator().manual_seed(seed)
    phrases = [torch.randint(0, vocabulary, (7,), generator=gen) for _ in range(5)]
    order = torch.randint(0, 5, (length // 7 + 2,), generator=gen)
    return torch.cat([phrases[i] for i in order])[:length].cuda()


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--vocabulary", type=int, default=500)
    p.add_argument("--width", type=int, default=128)
    p.add_argument("--heads", type=int, default=4)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--length", type=int, default=512)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    a = p.parse_args()
    model = TokenModel(a.vocabulary, a.width, a.heads, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    tokens = text(a.vocabulary, a.length + 1)
    inputs, targets = tokens[:-1], tokens[1:].clone()
    positions = torch.arange(a.length, device="cuda")
    # two documents, packed one behind the other; the first one's last token has no successor
    cut = a.length // 3
    starts = torch.tensor([0, cut, a.length], device="cuda")
    positions[cut:] -= cut
    targets[cut - 1] = -1
    for i in range(a.steps):
        loss, g = model.gradients(inputs, positions, targets, starts)
        size = torch.sqrt(sum(t.square().sum() for t in g.values()))
        model.step(g, 1.0 / max(1.0, float(size)))
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {float(loss):.4f}  gradient {float(size):.3f}", flush=True)
    state = model.new_state(1)
    prompt = inputs[:50]
    logp, entropy, ids, alternatives = model.read(prompt, positions[:50], state=state, targets=targets[:50], top=3)
    print(f"prompt of 50 tokens: mean log probability {float(logp.mean()):.4f}, entropy of the next token {float(entropy[-1]):.4f}")
    written = []
    following = ids[:1, -1]
    for i in range(12):
        written.append(int(following[0]))
        ids, alternatives, _ = model.write(following, torch.tensor([50 + i], device="cuda"), state)
        following = ids[0]
    print("written:", written)
    print("text:   ", inputs[50:62].tolist())


if __name__ == "__main__":
    main()
