#!/usr/bin/env python3
"""Training a network of gated blocks on token rows with approximate activations.

The method carried over to the blocks of language models: the forward pass is exact, what is kept for the backward pass are
block stores (8 or 4 bits a value and an eighth of a byte a block), and the gradients are computed from these.  A network
of L blocks on rows of C channels:

    n = w_pre * N(r)                                                  abl_resnorm_forward
    [g u] = n W1,  h = act(g) u,  b = h W2                            library products, abl_glu_forward
    r <- alpha r + beta gate * (w_post * N(b)),  n = w_pre * N(r)     abl_resnorm_forward

Per block and token it keeps the stores of N(b), N(r) (C values each) and of g, u (F values each); r and n live in two buffers
that all blocks share.  The backward pass of a block: dh = db W2^T, then abl_glu_backward makes [dg du] and the store of h, abl_ckpt_wgrad
the gradients of W2 (from that store) and W1 (from the store of N(r), scaled with w_pre), dn = [dg du] W1^T, and
abl_resnorm_backward carries dn and the residual stream's gradient to the block before.

    python -m paper_1901_07988_amd.token_blocks --layers 4 --tokens 2048 --channels 512 --width 1408 --steps 60

trains a student on a fixed teacher's outputs with exact storage (torch autograd on the same formulas), 8-bit and 4-bit stores from
the same initial parameters and batches, and prints the losses, the gradients' errors at the first step and what is kept per token.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B

EPS = 1e-5
PARAMETERS = ("W1", "W2", "gate", "w_post", "w_pre")
VECTORS = PARAMETERS[2:]


def random_parameters(layers, C, F, samples, seed):
    """One dict of fp32 tensors per block, and the last norm's weight.  gate: [samples, C]."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(shape, generator=gen, device="cuda") * std + mean

    blocks = [dict(W1=normal(C, 2 * F, std=C ** -0.5), W2=normal(F, C, std=F ** -0.5), gate=normal(samples, C, std=0.1, mean=0.7),
                   w_post=normal(C, std=0.1, mean=1.0), w_pre=normal(C, std=0.1, mean=1.0)) for _ in range(layers)]
    return blocks, normal(C, std=0.1, mean=1.0)


class TokenNet:
    """The network on `tokens` rows of bf16 with K-bit stores.  Rows come in `samples` runs of ceil(tokens / samples), the last one shorter, each
    with a row of every gate; where fewer runs hold all tokens, the gates' last rows are not used and their gradients are zero."""

    def __init__(self, parameters, w_last, tokens, K, act=B.ABL_ACT_SILU, alpha=1.0, beta=1.0):
        self.master, self.w_last32 = parameters, w_last
        C, F2 = parameters[0]["W1"].shape
        self.M, self.C, self.F, self.K, self.act = tokens, C, F2 // 2, K, act
        samples = parameters[0]["gate"].shape[0]
        self.gate_rows, self.alpha, self.beta = -(-tokens // samples), alpha, beta
        self.runs = -(-tokens // self.gate_rows)

        def tensor(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device="cuda")

        def store(width, k):
            return tensor(B.abl_ckpt_bytes(tokens, width, k), dtype=torch.uint8)

        f32 = torch.float32
        L = len(parameters)
        self.half = [{k: p[k].bfloat16() for k in PARAMETERS} for p in parameters]
        self.w_last = w_last.bfloat16()
        # kept for the backward pass: of the norm in front of each block (and the last one), of each block's gated unit and output
        self.norms = [dict(store=store(C, K), rstd=tensor(tokens, dtype=f32)) for _ in range(L + 1)]
        self.units = [dict(g=store(self.F, K), u=store(self.F, K)) for _ in range(L)]
        self.outputs = [dict(store=store(C, K), rstd=tensor(tokens, dtype=f32)) for _ in range(L)]
        # shared by all blocks
        self.r, self.n, self.b = tensor(tokens, C), tensor(tokens, C), tensor(tokens, C)
        self.gu, self.h = tensor(tokens, 2 * self.F), tensor(tokens, self.F)
        self.h_store = store(self.F, 8)
        self.grads = [{k: torch.zeros_like(p[k]) for k in PARAMETERS} for p in parameters]
        self.g_last = torch.zeros_like(w_last)
        self.earlier = []    # of a batch in several parts: the vectors' gradients of all parts but the last, per block; w_last's
        self.velocity = [{k: torch.zeros_like(p[k]) for k in PARAMETERS} for p in parameters]
        self.v_last = torch.zeros_like(w_last)
        self.scratch = tensor(max(B.abl_resnorm_scratch_bytes(tokens, C),
                                  B.abl_ckpt_wgrad_scratch_bytes(tokens, C, 2 * self.F, torch.bfloat16),
                                  B.abl_ckpt_wgrad_scratch_bytes(tokens, self.F, C, torch.bfloat16)), dtype=torch.uint8)

    def kept_bytes(self):
        """What waits for the backward pass."""
        return sum(t.numel() * t.element_size() for d in self.norms + self.units + self.outputs for t in d.values())

    def _w_pre(self, i):
        return self.half[i]["w_pre"] if i < len(self.half) else self.w_last

    def forward(self, x):
        """x [tokens, C] bf16 -> the last norm's output (valid until the next call)."""
        how = dict(K=self.K, eps=EPS)
        keep = self.norms[0]
        B.abl_resnorm_forward(x, None, None, 0, None, self._w_pre(0), self.r, self.n, ckpt_n=keep["store"], rstd_n=keep["rstd"], **how)
        for i, p in enumerate(self.half):
            torch.mm(self.n, p["W1"], out=self.gu)
            unit, out, keep = self.units[i], self.outputs[i], self.norms[i + 1]
            B.abl_glu_forward(self.gu[:, : self.F], self.gu[:, self.F:], self.h, self.act, self.K, unit["g"], unit["u"])
            torch.mm(self.h, p["W2"], out=self.b)
            B.abl_resnorm_forward(self.r, self.b, p["gate"][: self.runs], self.gate_rows, p["w_post"], self._w_pre(i + 1), self.r, self.n,
                                  ckpt_b=out["store"], rstd_b=out["rstd"], ckpt_n=keep["store"], rstd_n=keep["rstd"],
                                  alpha=self.alpha, beta=self.beta, **how)
        return self.n

    def backward(self, dn, accumulate=False):
        """dn: the loss gradient of forward's output.  Leaves every gradient in `grads` and `g_last`, returns the input's.
        accumulate: this is a further part of the last call's batch.  The products' gradients (W1, W2) are added to what is there; the others
        are this part's, those of the parts before wait in `earlier`, and `update` takes the sums."""
        if not accumulate:
            self.earlier = []
        elif self.earlier:
            for e, g in zip(self.earlier, self._vectors()):
                for k in e:
                    e[k] += g[k]
        else:
            self.earlier = [{k: g[k].clone() for k in g} for g in self._vectors()]
        flags = B.ABL_ACCUM_DW if accumulate else 0
        dr, db, dn = None, torch.empty_like(self.b), dn.clone()
        dgu, dh = torch.empty_like(self.gu), torch.empty_like(self.h)
        for i in reversed(range(len(self.half))):
            p, g, out, keep = self.half[i], self.grads[i], self.outputs[i], self.norms[i + 1]
            dr_new = dr if dr is not None else torch.empty_like(self.r)
            B.abl_resnorm_backward(dn, dr, p["gate"][: self.runs], self.gate_rows, p["w_post"], self._w_pre(i + 1), self.K, out["store"],
                                   out["rstd"], keep["store"], keep["rstd"], self.scratch, dr_new, db, g["gate"][: self.runs], g["w_post"],
                                   self._grad_pre(i + 1), self.alpha, self.beta)
            dr = dr_new
            torch.mm(db, p["W2"].t(), out=dh)
            unit = self.units[i]
            B.abl_glu_backward(dh, unit["g"], unit["u"], self.K, dgu[:, : self.F], dgu[:, self.F:], self.act, self.h_store)
            B.abl_ckpt_wgrad(self.h_store, 8, None, db, self.scratch, g["W2"], flags)
            B.abl_ckpt_wgrad(self.norms[i]["store"], self.K, self._w_pre(i), dgu, self.scratch, g["W1"], flags)
            torch.mm(dgu, p["W1"].t(), out=dn)
        keep = self.norms[0]
        B.abl_resnorm_backward(dn, dr, None, 0, None, self._w_pre(0), self.K, None, None, keep["store"], keep["rstd"], self.scratch,
                               dr, None, None, None, self._grad_pre(0), has_b=False)
        return dr

    def _vectors(self):
        return [{k: g[k] for k in VECTORS} for g in self.grads] + [{"w_last": self.g_last}]

    def _grad_pre(self, i):
        return self.grads[i]["w_pre"] if i < len(self.grads) else self.g_last

    def update(self, lr, momentum=0.9, weight_decay=0.0):
        """SGD on the fp32 parameters, and their bf16 copies."""
        for i, (p, g, v, h) in enumerate(zip(self.master, self.grads, self.velocity, self.half)):
            for k in PARAMETERS:
                d = g[k] + self.earlier[i][k] if self.earlier and k in VECTORS else g[k]
                B.abl_sgd_momentum(p[k].view(-1), d.view(-1), v[k].view(-1), lr, momentum, weight_decay)
                h[k].copy_(p[k])
        d = self.g_last + self.earlier[-1]["w_last"] if self.earlier else self.g_last
        B.abl_sgd_momentum(self.w_last32, d, self.v_last, lr, momentum, weight_decay)
        self.w_last.copy_(self.w_last32)


class ExactNet:
    """The same network with everything kept: the formulas in fp32 on bf16 parameters, gradients by torch's autograd."""

    def __init__(self, parameters, w_last, tokens, act=B.ABL_ACT_SILU, alpha=1.0, beta=1.0):
        self.master, self.w_last32, self.alpha, self.beta, self.act = parameters, w_last, alpha, beta, act
        self.M = tokens
        self.gate_rows = -(-tokens // parameters[0]["gate"].shape[0])
        self.velocity = [{k: torch.zeros_like(p[k]) for k in PARAMETERS} for p in parameters]
        self.v_last = torch.zeros_like(w_last)

    @staticmethod
    def _norm(x):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)

    def forward(self, x):
        self.leaves = [{k: p[k].bfloat16().float().requires_grad_() for k in PARAMETERS} for p in self.master]
        self.last = self.w_last32.bfloat16().float().requires_grad_()
        r = x.float()
        for p in self.leaves:
            g, u = (self._norm(r) * p["w_pre"] @ p["W1"]).chunk(2, -1)
            a = torch.nn.functional.silu(g) if self.act == B.ABL_ACT_SILU else torch.nn.functional.gelu(g, approximate="tanh")
            gate = p["gate"].repeat_interleave(self.gate_rows, 0)[: self.M]
            r = self.alpha * r + self.beta * gate * (p["w_post"] * self._norm(a * u @ p["W2"]))
        self.out = self._norm(r) * self.last
        return self.out

    def backward(self, dn):
        leaves = [t for p in self.leaves for t in p.values()] + [self.last]
        grads = list(torch.autograd.grad(self.out, leaves, dn.float()))
        self.g_last = grads.pop()
        self.grads = [{k: grads.pop(0) for k in p} for p in self.leaves]

    def update(self, lr, momentum=0.9, weight_decay=0.0):
        for p, g, v in zip(self.master, self.grads, self.velocity):
            for k in PARAMETERS:
                B.abl_sgd_momentum(p[k].view(-1), g[k].contiguous().view(-1), v[k].view(-1), lr, momentum, weight_decay)
        B.abl_sgd_momentum(self.w_last32, self.g_last.contiguous(), self.v_last, lr, momentum, weight_decay)


def batch(tokens, C, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(tokens, C, generator=gen, device="cuda").bfloat16()


def relative(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


def gradient_errors(net, exact):
    """{name: relative error of net's gradients against the exact ones', over all blocks}."""
    return {k: max(relative(a[k], b[k]) for a, b in zip(net.grads, exact.grads)) for k in PARAMETERS}


def train(make, teacher, tokens, C, steps, lr, seed=1000):
    net, losses = make(), []
    for s in range(steps):
        x = batch(tokens, C, seed + s)
        target = teacher.forward(x).detach().float().clone()
        diff = net.forward(x).detach().float() - target
        losses.append(float((diff * diff).mean()) / 2)
        net.backward((diff / tokens).bfloat16())
        net.update(lr)
    return losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--samples", type=int, default=4)
    ap.add_argument("--channels", type=int, default=512)
    ap.add_argument("--width", type=int, default=1408)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=0.02)
    a = ap.parse_args(argv)
    size = (a.layers, a.channels, a.width, a.samples)
    teacher = ExactNet(*random_parameters(*size, seed=7), a.tokens)
    fresh = lambda: random_parameters(*size, seed=8)  # noqa: E731
    curves = {"exact": train(lambda: ExactNet(*fresh(), a.tokens), teacher, a.tokens, a.channels, a.steps, a.lr)}
    for K in (8, 4):
        curves["K=%d" % K] = train(lambda: TokenNet(*fresh(), a.tokens, K), teacher, a.tokens, a.channels, a.steps, a.lr)
    print("step     " + "  ".join("%-9s" % k for k in curves))
    for s in range(0, a.steps, max(1, a.steps // 10)):
        print("%-8d " % s + "  ".join("%-9.5f" % c[s] for c in curves.values()), flush=True)
    x, dn = batch(a.tokens, a.channels, 1), batch(a.tokens, a.channels, 2)
    exact = ExactNet(*fresh(), a.tokens)
    exact.forward(x)
    exact.backward(dn)
    for K in (8, 4):
        net = TokenNet(*fresh(), a.tokens, K)
        net.forward(x)
        net.backward(dn)
        print("K=%d: %.0f bytes kept per token (bf16 tensors: %.0f), gradient errors %s" % (
            K, net.kept_bytes() / a.tokens, 2 * (a.channels * (2 * a.layers + 1) + 2 * a.layers * a.width),
            ", ".join("%s %.4f" % kv for kv in gradient_errors(net, exact).items())), flush=True)
    return curves


if __name__ == "__main__":
    main()
