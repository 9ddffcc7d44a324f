#!/usr/bin/env python3
"""A vocabulary behind the network of gated blocks (token_blocks.py): its last norm's rows against a table of tokens, trained on labels and on a
teacher's largest logits.

    loss = label_weight CE + teacher_weight KD, the mean over the rows (all count here)  abl_xent_forward, abl_distill_forward
    dn, dTable                                                                            abl_xent_backward, abl_distill_backward

The logits are never kept: what waits for the backward pass beside the blocks' stores is a row's log-sums and, with a teacher, its logits
at the teacher's tokens.  The last norm's output is still in the network's buffer then.

    python -m paper_1901_07988_amd.token_head --layers 2 --tokens 2048 --channels 256 --width 704 --vocab 1024 --top 16 --steps 300

trains students of the same initial parameters on a fixed teacher's most likely tokens: on these as labels, on its largest logits at a
temperature, and on both, with 8-bit stores, and prints the cross entropy on fresh rows and what is kept per token.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from .token_blocks import ExactNet, TokenNet, batch, random_parameters


class VocabularyHead:
    """Table [V, C] behind `tokens` rows of C channels.  top: entries of a row that a teacher gives (0: labels only)."""

    def __init__(self, table, tokens, top=0, temperature=1.0, label_weight=1.0, teacher_weight=1.0, smoothing=0.0, z_weight=0.0):
        self.master = table
        assert top or (temperature, label_weight, teacher_weight) == (1.0, 1.0, 1.0), "labels alone have neither a temperature nor weights"
        V, C = table.shape
        self.M, self.V, self.C, self.T = tokens, V, C, top
        self.how = dict(smoothing=smoothing, z_weight=z_weight)
        if top:
            self.how |= dict(temperature=temperature, label_weight=label_weight, teacher_weight=teacher_weight)
        self.half = table.bfloat16()

        def numbers(*shape):
            return torch.empty(shape, device="cuda")

        self.loss, self.lse = numbers(tokens), numbers(tokens)
        self.lse_t, self.z_top = (numbers(tokens), numbers(tokens, top)) if top else (None, None)
        self.grad, self.velocity = torch.zeros_like(table), torch.zeros_like(table)
        size = dict(T=top, dw_dtype=torch.float32)
        self.scratch = torch.empty(max(B.abl_head_scratch_bytes(tokens, C, V, torch.bfloat16, backward=back, **size) for back in (False, True)),
                                   dtype=torch.uint8, device="cuda")

    def kept_bytes(self):
        """What waits for the backward pass."""
        return sum(t.numel() * 4 for t in (self.lse, self.lse_t, self.z_top) if t is not None)

    def forward(self, n, labels, ids=None, logits=None):
        """n [tokens, C] bf16 -> the rows' losses (valid until the next call; zero where a row does not count)."""
        if self.T:
            B.abl_distill_forward(n, self.half, labels, ids, logits, self.scratch, self.loss, self.lse, self.lse_t, self.z_top, **self.how)
        else:
            B.abl_xent_forward(n, self.half, labels, self.scratch, self.loss, self.lse, **self.how)
        return self.loss

    def backward(self, n, labels, dloss, ids=None, logits=None, accumulate=False):
        """dloss: the gradient of every row's loss.  Returns the gradient of n, leaves the table's in `grad`."""
        dn, flags = torch.empty_like(n), B.ABL_ACCUM_DW if accumulate else 0
        if self.T:
            B.abl_distill_backward(n, self.half, labels, ids, logits, self.lse, self.lse_t, self.z_top, dloss, self.scratch, dn, self.grad, flags=flags,
                                   **self.how)
        else:
            B.abl_xent_backward(n, self.half, labels, self.lse, dloss, self.scratch, dn, self.grad, flags=flags, **self.how)
        return dn

    def update(self, lr, momentum=0.9, weight_decay=0.0):
        B.abl_sgd_momentum(self.master.view(-1), self.grad.view(-1), self.velocity.view(-1), lr, momentum, weight_decay)
        self.half.copy_(self.master)


class Teacher:
    """A fixed network with a table: its most likely tokens and its largest logits."""

    def __init__(self, layers, C, F, samples, V, tokens, seed):
        self.net = ExactNet(*random_parameters(layers, C, F, samples, seed=seed), tokens)
        self.table = random_table(V, C, seed + 1)

    def look(self, x, top):
        z = self.net.forward(x).detach() @ self.table.t()
        best = torch.topk(z, top)
        return best.indices[:, 0].contiguous(), best.indices, best.values.float()


def random_table(V, C, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(V, C, generator=gen, device="cuda") * (4 * C ** -0.5)


def train(net, head, teacher, top, steps, lr, seed=1000):
    tokens, C = net.M, net.C
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    losses = []
    for s in range(steps):
        x = batch(tokens, C, seed + s)
        labels, ids, logits = teacher.look(x, max(top, 1))
        extra = (ids, logits) if head.T else ()
        n = net.forward(x)
        losses.append(float(head.forward(n, labels, *extra).mean()))
        net.backward(head.backward(n, labels, weight, *extra))
        net.update(lr)
        head.update(lr)
    return losses


def cross_entropy(net, table, teacher, tokens, C, seed=99):
    x = batch(tokens, C, seed)
    labels, _, _ = teacher.look(x, 1)
    head = VocabularyHead(table, tokens)
    return float(head.forward(net.forward(x), labels).mean())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--samples", type=int, default=4)
    ap.add_argument("--channels", type=int, default=256)
    ap.add_argument("--width", type=int, default=704)
    ap.add_argument("--vocab", type=int, default=1024)
    ap.add_argument("--top", type=int, default=16)
    ap.add_argument("--temperature", type=float, default=2.0)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--lr", type=float, default=0.1)
    a = ap.parse_args(argv)
    C, V = a.channels, a.vocab
    teacher = Teacher(a.layers, C, a.width, a.samples, V, a.tokens, seed=7)
    students = {"labels": dict(top=0), "logits": dict(top=a.top, temperature=a.temperature, label_weight=0.0),
                "both": dict(top=a.top, temperature=a.temperature, label_weight=0.5, teacher_weight=0.5)}
    curves, after = {}, {}
    for name, how in students.items():
        net = TokenNet(*random_parameters(a.layers, C, a.width, a.samples, seed=8), a.tokens, 8)
        head = VocabularyHead(random_table(V, C, 9), a.tokens, **how)
        curves[name] = train(net, head, teacher, a.top, a.steps, a.lr)
        after[name] = cross_entropy(net, head.master, teacher, a.tokens, C)
        print("%-6s loss %.4f -> %.4f, cross entropy on fresh rows %.4f; kept per token: blocks %.0f bytes, head %.0f (logits: %d)" % (
            name, curves[name][0], curves[name][-1], after[name], net.kept_bytes() / a.tokens, head.kept_bytes() / a.tokens, 4 * V), flush=True)
    return curves, after


if __name__ == "__main__":
    main()
