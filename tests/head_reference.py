"""The losses over a vocabulary in 64 bits, from their definition, with bounds on what the GPU's arithmetic may add: every rounding is
counted with half a step of its type (bf16 2^-8, fp32 2^-24, relative to the value)."""
import math

import torch

B16, F32 = 2.0 ** -8, 2.0 ** -24
F64 = torch.float64


class Settings:
    def __init__(self, scale=1.0, smoothing=0.0, z_weight=0.0, temperature=1.0, label_weight=1.0, teacher_weight=0.0):
        self.scale, self.smoothing, self.z_weight = scale, smoothing, z_weight
        self.tau, self.lw, self.kw = temperature, label_weight, teacher_weight


def _teacher(ids, t, n, V):
    """Dense rows of the teacher's probabilities (double), the entropy term, which rows have entries, which entries are there."""
    there = (ids >= 0) & ~(t == -math.inf)
    u = torch.where(there, t.to(F64) / n.tau, torch.full_like(t, -math.inf, dtype=F64))
    has = there.any(1)
    p = torch.zeros_like(u)
    p[has] = torch.softmax(u[has], 1)
    dense = torch.zeros(ids.shape[0], V, dtype=F64)
    r, k = there.nonzero(as_tuple=True)
    ok = ids[r, k] < V
    dense.index_put_((r[ok], ids[r, k][ok]), p[r, k][ok], accumulate=True)
    return p, dense, torch.special.xlogy(p, p).sum(1), has, there


def forward(h, W, labels, n, ids=None, t=None):
    """Everything on the CPU.  dict of loss, lse, (lse_t, z_top,) and `bound`, the same with what the kernels' results may be off."""
    h, W = h.to(F64), W.to(F64)
    M, V = h.shape[0], W.shape[0]
    counts = torch.zeros(M, dtype=torch.bool) if labels is None else labels >= 0
    if ids is not None:
        p, dense, entropy, has, there = _teacher(ids, t, n, V)
        counts = counts | has
    h = torch.where(counts[:, None], h, torch.zeros((), dtype=F64))
    z = n.scale * (h @ W.t())
    ez = logit_bound(h, W, n)
    L, Lt = torch.logsumexp(z, 1), torch.logsumexp(z / n.tau, 1)
    # of a log-sum: the largest error of a logit; the sum's roundings, one after the other (a lane's share, its tile's, the tiles'), and each
    # term's: the exponent's argument |z - top| <= 100 to half a step, twice, and the instructions' last bits
    eL = ez.amax(1) + (V / 64 + 300) * F32 + 4 * F32 * L.abs() + 2.0 ** -18 * (z.amax(1) - z.amin(1) > 16) + 2.0 ** -20
    loss, el = n.z_weight * L * L, 2 * abs(n.z_weight) * L.abs() * eL + 4 * F32 * (n.z_weight * L * L).abs()
    if labels is not None:
        has_y = labels >= 0
        y = labels.clamp(0, V - 1)
        zy = z.gather(1, y[:, None])[:, 0]
        ce = (1 - n.smoothing) * (L - zy) + n.smoothing * (L - z.mean(1))
        e = eL + ez.amax(1) + (V / 64 + 300) * F32 * z.abs().mean(1) * n.smoothing + 8 * F32 * (L.abs() + z.abs().amax(1))
        loss = loss + torch.where(has_y, n.lw * ce, torch.zeros_like(ce))
        el = el + abs(n.lw) * e
    out, bound = {}, {}
    if ids is not None:
        kd = n.tau ** 2 * (entropy + (dense * (Lt[:, None] - z / n.tau)).sum(1))
        size = 1 + Lt.abs() + z.abs().amax(1) / n.tau + torch.where(there & (t == t), t.to(F64).abs(), torch.zeros((), dtype=F64)).amax(1) / n.tau
        loss = loss + torch.where(has, n.kw * kd, torch.zeros_like(kd))
        el = el + abs(n.kw) * n.tau ** 2 * (2 * eL + (ids.shape[1] / 16 + 60) * F32 * size)
        safe = ids.clamp(0, V - 1)
        out = dict(lse_t=torch.where(counts, Lt, torch.zeros_like(Lt)), z_top=torch.where(there, z.gather(1, safe), torch.zeros((), dtype=F64)))
        bound = dict(lse_t=eL + 8 * F32 * z.abs().amax(1), z_top=ez.gather(1, safe))
    zero = torch.zeros_like(loss)
    out |= dict(loss=torch.where(counts, loss, zero), lse=torch.where(counts, L, zero))
    bound |= dict(loss=el + 8 * F32 * loss.abs(), lse=eL)
    return out | dict(bound=bound)


def logit_bound(h, W, n):
    """Products of bf16 are exact in fp32; of fp32 in parts they lack 2^-23 (parts left out); C + 64 roundings of sums, the scale's."""
    return (h.shape[1] + 70) * F32 * abs(n.scale) * (h.abs() @ W.abs().t()) + 1e-37


def backward(h, W, labels, lse, dloss, n, type, dw_type, one_part=False, ids=None, t=None, lse_t=None):
    """dict of dh, dW and `bound`: from the log-sums as they are given (fp32 values)."""
    h, W, lse, w = h.to(F64), W.to(F64), lse.to(F64), dloss.to(F64) * n.scale
    M, V = h.shape[0], W.shape[0]
    zero = torch.zeros((), dtype=F64)
    labelled = torch.zeros(M, dtype=torch.bool) if labels is None else labels >= 0
    hard = torch.zeros(M, V, dtype=F64)
    if labels is not None:
        r = labelled.nonzero()[:, 0]
        hard[r, labels[r]] = 1 - n.smoothing
        hard[r] += n.smoothing / V
    counts, taught, soft = labelled, torch.zeros_like(labelled), 0.0
    if ids is not None:
        _, soft, _, taught, _ = _teacher(ids, t, n, V)
        counts = labelled | taught
    h = torch.where(counts[:, None], h, zero)
    z, ez = n.scale * (h @ W.t()), logit_bound(h, W, n)
    q = torch.exp(z - lse[:, None])
    on = n.lw * labelled[:, None] + 2 * n.z_weight * lse[:, None]
    d, size = on * q - n.lw * hard, on.abs() * q * (ez + 2.0 ** -20 + 4 * F32 * (z - lse[:, None]).abs()) + 8 * F32 * n.lw * hard.abs()
    if ids is not None:
        qt = torch.exp(z / n.tau - lse_t.to(F64)[:, None]) * taught[:, None]
        d = d + n.kw * n.tau * (qt - soft)
        size = size + abs(n.kw) * n.tau * (qt * (ez / n.tau + 2.0 ** -20 + 6 * F32 * (z / n.tau - lse_t.to(F64)[:, None]).abs()) +
                                           (ids.shape[1] / 16 + 80) * F32 * (1 + t.to(F64).abs().where(t > -math.inf, zero).amax(1, keepdim=True) / n.tau) * soft)
    w = torch.where(counts, w, zero)[:, None]
    d, size = d * w, size * w.abs() + 4 * F32 * (d * w).abs()
    # the gradient of the logits in parts of 8 bits, each rounded
    parts = 1 if one_part else 3 if torch.float32 in (type, dw_type) else 1
    lost = {1: B16, 3: B16 ** 3}
    ed_h = size + lost[1 if type == torch.bfloat16 else parts] * d.abs()
    ed_w = size + lost[parts] * d.abs()
    dh, dW = d @ W, d.t() @ h
    half = {torch.bfloat16: B16, torch.float32: F32}
    b_h = ed_h @ W.abs() + (V + 70) * F32 * (d.abs() @ W.abs()) + half[type] * dh.abs()
    b_w = ed_w.t() @ h.abs() + (M + 70) * F32 * (d.abs().t() @ h.abs()) + half[dw_type] * dW.abs()
    return dict(dh=dh, dW=dW, bound=dict(dh=1.01 * b_h + 1e-37, dW=1.01 * b_w + 1e-37))


def assert_within(got, want, bound, name):
    got, bound = got.detach().cpu().to(F64), bound.expand_as(want)
    off = (got - want).abs()
    worst = int((off - bound).argmax())
    assert bool((off <= bound).all()), "%s: %g off at %d (%g), %g allowed" % (
        name, off.flatten()[worst], worst, want.flatten()[worst], bound.flatten()[worst])
