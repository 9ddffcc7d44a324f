"""The losses behind the last block of a language model, as measurable cases: what a network's rows are worth against a vocabulary,
without the logits being kept.

  xent_fwd     cross entropy of rows h [M, C] against a table W [V, C]: loss and log-sum of every row
  xent_bwd     the gradients of h and W, from the log-sums and the gradient of every row's loss
  distill_fwd  distillation from the T largest logits of a teacher, alone or next to the cross entropy
  distill_bwd  its gradients

With z = scale h W^T, L = log sum_v exp z_v, L_t = log sum_v exp(z_v / tau), a row's label y and the teacher's entries (i_k, t_k):

  CE = (1 - smoothing) (L - z_y) + smoothing (L - mean_v z_v)
  KD = tau^2 sum_k p_k (log p_k - z_{i_k} / tau + L_t),  p = softmax of t / tau over the row's entries
  xent     loss = CE + z_weight L^2
  distill  loss = label_weight CE + z_weight L^2 + teacher_weight KD

A label below zero is none, an entry with an id below zero or a logit of minus infinity is absent.  A row without a label and without
entries does not count: its loss, log-sums and gradient are zero.  A row with entries but no label has no CE, one without entries no KD.
"""
import math

import torch

own = False
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MAX_PRODUCT = 8192 * 4096 * 65536
CHUNK = 1 << 28    # logits that are made at a time where inputs are prepared


# ---- the cases ----------------------------------------------------------------------------------------
def xent(op, M, C, V, type, dw="bf16", ignored=0.0, smoothing=0.0, z_weight=0.0, scale=1.0, pitch=0):
    """dw: the type of the table's gradient; ignored: share of the rows without a label; pitch: h and W are column slices of tensors
    that are so many channels wider."""
    return dict(op=op, M=M, C=C, V=V, type=type, dw=dw, ignored=ignored, smoothing=smoothing, z_weight=z_weight, scale=scale, pitch=pitch)


def distill(op, M, C, V, T, type, dw="bf16", tau=1.0, label_weight=0.0, ignored=0.0, z_weight=0.0, pitch=0):
    return dict(op=op, M=M, C=C, V=V, T=T, type=type, dw=dw, tau=tau, label_weight=label_weight, ignored=ignored, z_weight=z_weight, pitch=pitch)


def listed():
    return [
        # serving: the log-probability of one sequence's next token, small network: the smallest call
        dict(xent("xent_fwd", 1, 1024, 32768, "bf16"), name="xent_fwd_one_token"),
        # scoring: one new token of each of sixteen sequences, the table of a large vocabulary
        dict(xent("xent_fwd", 16, 4096, 131072, "bf16"), name="xent_fwd_serve"),
        # training, the largest: four sequences of 2048 tokens
        dict(xent("xent_fwd", 8192, 4096, 65536, "bf16"), name="xent_fwd_train"),
        dict(xent("xent_bwd", 8192, 4096, 65536, "bf16"), name="xent_bwd_train"),
        # fine-tuning: six rows of ten are prompts and padding; smoothed labels, a penalty on the log-sum, the table's gradient in fp32 (it is added up)
        dict(xent("xent_bwd", 8192, 2048, 32768, "bf16", dw="f32", ignored=0.6, smoothing=0.1, z_weight=1e-4), name="xent_bwd_prompts"),
        # sizes that no tile divides, in fp32; slices of wider tensors
        dict(xent("xent_fwd", 1500, 1111, 5003, "f32", dw="f32", ignored=0.2, smoothing=0.1, scale=0.5, pitch=9), name="xent_fwd_odd_f32"),
        dict(xent("xent_bwd", 1500, 1111, 5003, "f32", dw="f32", ignored=0.2, smoothing=0.1, scale=0.5, pitch=9), name="xent_bwd_odd_f32"),
        # a short ragged batch on a small table
        dict(xent("xent_bwd", 61, 1000, 1013, "bf16"), name="xent_bwd_small"),
        # a student's loss on a handful of tokens
        dict(distill("distill_fwd", 16, 2048, 32768, 8, "bf16"), name="distill_fwd_small"),
        # training a student on the 32 largest logits of a large vocabulary, softened, next to the labels
        dict(distill("distill_fwd", 4096, 2048, 131072, 32, "bf16", tau=2.0, label_weight=0.5, ignored=0.3), name="distill_fwd_train"),
        dict(distill("distill_bwd", 4096, 2048, 131072, 32, "bf16", tau=2.0, label_weight=0.5, ignored=0.3), name="distill_bwd_train"),
        # odd sizes in fp32, the teacher alone
        dict(distill("distill_bwd", 700, 1000, 10007, 5, "f32", dw="f32", tau=4.0, ignored=0.1), name="distill_bwd_odd_f32"),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, min(hi, v))

    def even(v, step):
        return v if rng.random() < 0.4 else max(step, v // step * step)

    op = rng.choice(["xent_fwd", "xent_bwd", "distill_fwd", "distill_bwd"])
    type = rng.choice(["f32", "bf16", "bf16"])
    C, V = even(size(64, 8192), 64), even(size(100, 131072), 128)
    M = size(1, 8192)
    most = MAX_PRODUCT // (1 if type == "bf16" else 8)
    M = max(1, min(M, most // (C * V)))
    dw = type if type == "f32" else rng.choice(["bf16", "bf16", "f32"])
    common = dict(dw=dw, ignored=rng.choice([0.0, 0.0, 0.3, 0.9]), z_weight=rng.choice([0.0, 1e-4]), pitch=rng.choice([0, 0, 8, 37]))
    if op.startswith("xent"):
        return xent(op, M, C, V, type, smoothing=rng.choice([0.0, 0.1]), scale=rng.choice([1.0, 0.25]), **common)
    return distill(op, M, C, V, min(V, size(1, 64)), type, tau=rng.choice([1.0, 1.0, 2.0, 4.0]), label_weight=rng.choice([0.0, 0.5, 1.0]), **common)


# ---- inputs -------------------------------------------------------------------------------------------
def settings(c):
    """The numbers of the formulas above that a case leaves at what its operator takes for them."""
    if c["op"].startswith("xent"):
        return dict(scale=c["scale"], smoothing=c["smoothing"], z_weight=c["z_weight"], tau=1.0, label_weight=1.0, teacher_weight=0.0)
    return dict(scale=1.0, smoothing=0.0, z_weight=c["z_weight"], tau=c["tau"], label_weight=c["label_weight"], teacher_weight=1.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c = dict(case)
    T, M, C, V, op = TYPES[c["type"]], c["M"], c["C"], c["V"], c["op"]

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def tensor(*shape, dtype=T):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = dict(case=c)
    s["W"] = (normal(V, C + c["pitch"]) * C ** -0.5).to(T)[:, :C]
    # labels: small ids are the frequent ones; the network leans towards the right token, more or less
    labels = (torch.exp(uniform(M) * math.log(V + 1)) - 1).long().clamp(max=V - 1)
    h = normal(M, C + c["pitch"])
    h[:, :C] += 6 * uniform(M, 1) * s["W"][labels].float()
    s["h"] = (h * (2.0 / c.get("scale", 1.0))).to(T)[:, :C]
    counts = uniform(M) >= c["ignored"]
    counts[0] = True
    s["labels"] = torch.where(counts, labels, -100)
    if op.startswith("distill"):
        K = c["T"]
        # the teacher knows the label better than the student and sees the rest much as it does
        ids, logits = tensor(M, K, dtype=torch.int64), tensor(M, K, dtype=torch.float32)
        step = max(1, CHUNK // V)
        wt = s["W"].t()
        for m in range(0, M, step):
            t = (s["h"][m: m + step] @ wt).float()
            t += normal(*t.shape)
            t.scatter_(1, labels[m: m + step, None], t.amax(1, keepdim=True) + 2)
            t = torch.topk(t, K)
            logits[m: m + step], ids[m: m + step] = t.values, t.indices
        # prompts have no entries either; some rows have fewer than the others
        few = (uniform(M) * 4 * K).long().clamp(min=1)
        there = counts[:, None] & (torch.arange(K, device="cuda")[None] < few[:, None])
        s["top_ids"], s["top_logits"] = torch.where(there, ids, -1), logits
        if not c["label_weight"]:
            s["labels"] = None
        s["lse_t"], s["z_top"] = tensor(M, dtype=torch.float32), tensor(M, K, dtype=torch.float32)
    s["loss"], s["lse"] = tensor(M, dtype=torch.float32), tensor(M, dtype=torch.float32)
    if op.endswith("bwd"):
        kept = forward(s)
        s["lse"] = kept["lse"]
        if op.startswith("distill"):
            s["lse_t"], s["z_top"] = kept["lse_t"], kept["z_top"]
        s["dloss"] = torch.full((M,), 1.0 / max(1, M), device="cuda") * (0.5 + uniform(M))
        s["dh"], s["dW"] = tensor(M, C), tensor(V, C, dtype=TYPES[c["dw"]])
    if own:
        from paper_1901_07988_amd import binding as B
        n = B.abl_head_scratch_bytes(M, C, V, T, T=c.get("T", 0), dw_dtype=TYPES[c["dw"]], backward=op.endswith("bwd"))
        s["scratch"] = tensor(n, dtype=torch.uint8)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------
def logits_of(s, scale):
    return (s["h"].float() @ s["W"].float().t()) * scale


def log_sum(z):
    top = z.amax(1)
    return top + torch.log(torch.exp(z - top[:, None]).sum(1))


def teacher_of(s, tau):
    """(probabilities [M, T], whether an entry is there, ids that can be looked up)"""
    t = s["top_logits"] / tau
    there = (s["top_ids"] >= 0) & (t > -math.inf)
    t = torch.where(there, t, -math.inf)
    top = t.amax(1, keepdim=True)
    e = torch.where(there, torch.exp(t - torch.where(top > -math.inf, top, 0.0)), 0.0)
    return e / e.sum(1, keepdim=True).clamp(min=1e-30), there, s["top_ids"].clamp(min=0)


def forward(s):
    c = s["case"]
    n = settings(c)
    z = logits_of(s, n["scale"])
    L = log_sum(z)
    out, loss = {}, torch.zeros_like(L)
    counts = torch.zeros_like(L, dtype=torch.bool)
    if s["labels"] is not None:
        has, y = s["labels"] >= 0, s["labels"].clamp(min=0)
        ce = L - z.gather(1, y[:, None])[:, 0]
        if n["smoothing"]:
            ce = (1 - n["smoothing"]) * ce + n["smoothing"] * (L - z.mean(1))
        loss = torch.where(has, n["label_weight"] * ce, loss)
        counts = has
    if c["op"].startswith("distill"):
        tau = n["tau"]
        p, there, ids = teacher_of(s, tau)
        has = there.any(1)
        z_top = torch.where(there, z.gather(1, ids), 0.0)
        lse_t = log_sum(z / tau) if tau != 1 else L
        kd = (p * (torch.log(p.clamp(min=1e-30)) - z_top / tau + lse_t[:, None])).sum(1) * tau ** 2
        loss = loss + torch.where(has, n["teacher_weight"] * kd, 0.0)
        counts = counts | has
        out = dict(lse_t=torch.where(counts, lse_t, 0.0), z_top=z_top)
    if n["z_weight"]:
        loss = loss + n["z_weight"] * L * L
    return dict(loss=torch.where(counts, loss, 0.0), lse=torch.where(counts, L, 0.0)) | out


def backward(s):
    c = s["case"]
    n = settings(c)
    z, w = logits_of(s, n["scale"]), s["dloss"] * n["scale"]
    lse = s["lse"]
    on_q, on_qt = torch.zeros_like(w), torch.zeros_like(w)
    counts = torch.zeros_like(w, dtype=torch.bool)
    if s["labels"] is not None:
        counts = s["labels"] >= 0
        on_q = torch.where(counts, w * n["label_weight"], 0.0)
    if c["op"].startswith("distill"):
        p, there, ids = teacher_of(s, n["tau"])
        has = there.any(1)
        counts = counts | has
        on_qt = torch.where(has, w * n["teacher_weight"] * n["tau"], 0.0)
    if n["z_weight"]:
        on_q = on_q + torch.where(counts, 2 * n["z_weight"] * w * lse, 0.0)
    dz = torch.exp(z - lse[:, None]) * on_q[:, None]
    if c["op"].startswith("distill"):
        dz = dz + torch.exp(z / n["tau"] - s["lse_t"][:, None]) * on_qt[:, None]
        dz.scatter_add_(1, ids, -p * on_qt[:, None])
    if s["labels"] is not None:
        has, y = s["labels"] >= 0, s["labels"].clamp(min=0)
        weight = torch.where(has, w * n["label_weight"], 0.0)
        if n["smoothing"]:
            dz = dz - (weight * (n["smoothing"] / c["V"]))[:, None]
        dz.scatter_add_(1, y[:, None], -(weight * (1 - n["smoothing"]))[:, None])
    dz = torch.where(counts[:, None], dz, 0.0)
    h = torch.where(counts[:, None], s["h"].float(), 0.0)
    return dict(dh=(dz @ s["W"].float()).to(TYPES[c["type"]]), dW=(dz.t() @ h).to(TYPES[c["dw"]]))


def plain(s):
    if s["case"]["op"].endswith("bwd"):
        return backward(s)
    return forward(s)


# ---- the framework's calls ----------------------------------------------------------------------------
def run(s):
    if not own:
        return plain(s)
    from paper_1901_07988_amd import binding as B
    c, n = s["case"], settings(s["case"])
    op = c["op"]
    how = dict(scale=n["scale"], smoothing=n["smoothing"], z_weight=n["z_weight"])
    if op == "xent_fwd":
        B.abl_xent_forward(s["h"], s["W"], s["labels"], s["scratch"], s["loss"], s["lse"], **how)
        return dict(loss=s["loss"], lse=s["lse"])
    if op == "xent_bwd":
        B.abl_xent_backward(s["h"], s["W"], s["labels"], s["lse"], s["dloss"], s["scratch"], s["dh"], s["dW"], **how)
        return dict(dh=s["dh"], dW=s["dW"])
    how |= dict(temperature=n["tau"], label_weight=n["label_weight"], teacher_weight=n["teacher_weight"])
    if op == "distill_fwd":
        B.abl_distill_forward(s["h"], s["W"], s["labels"], s["top_ids"], s["top_logits"], s["scratch"], s["loss"], s["lse"], s["lse_t"],
                              s["z_top"], **how)
        return dict(loss=s["loss"], lse=s["lse"], lse_t=s["lse_t"], z_top=s["z_top"])
    B.abl_distill_backward(s["h"], s["W"], s["labels"], s["top_ids"], s["top_logits"], s["lse"], s["lse_t"], s["z_top"], s["dloss"],
                           s["scratch"], s["dh"], s["dW"], **how)
    return dict(dh=s["dh"], dW=s["dW"])


def work(case):
    c = case
    M, C, V, K = c["M"], c["C"], c["V"], c.get("T", 0)
    t, d = (4 if c["type"] == "f32" else 2), (4 if c["dw"] == "f32" else 2)
    rows = max(1, round(M * (1 - c["ignored"])))     # that count
    b = rows * C * t + V * C * t + M * 8 + M * K * 12
    if c["op"].endswith("fwd"):
        return dict(bytes=b + M * 8 + (M * (4 + 4 * K) if K else 0), flops=2 * rows * C * V)
    return dict(bytes=b + M * 8 + (M * (4 + 4 * K) if K else 0) + M * C * t + V * C * d, flops=6 * rows * C * V)


# ---- the definition in 64 bits ------------------------------------------------------------------------
def exact(case, seed):
    """A band of rows at a time; each row's distribution from its own logits, targets as dense rows."""
    s = prepare(case, seed)
    c = s["case"]
    M, V = c["M"], c["V"]
    n = settings(c)
    tau, zw, lw, kw, eps = n["tau"], n["z_weight"], n["label_weight"], n["teacher_weight"], n["smoothing"]
    teacher, back = c["op"].startswith("distill"), c["op"].endswith("bwd")
    W = s["W"].double().contiguous()
    f64 = dict(dtype=torch.float64, device="cuda")
    parts = []
    dW = torch.zeros(W.shape, **f64) if back else None
    step = max(1, CHUNK // V)
    for m in range(0, M, step):
        h = s["h"][m: m + step].double().contiguous()
        R = h.shape[0]
        z = n["scale"] * torch.mm(h, W.t())
        hard = torch.zeros(R, V, **f64)                    # the label's row
        labelled = torch.zeros(R, dtype=torch.bool, device="cuda")
        if s["labels"] is not None:
            y = s["labels"][m: m + step]
            labelled = y >= 0
            r = labelled.nonzero()[:, 0]
            hard[r, y[r]] = 1.0 - eps
            hard[r] += eps / V
        taught = torch.zeros_like(labelled)
        if teacher:
            ids, t = s["top_ids"][m: m + step], s["top_logits"][m: m + step].double() / tau
            there = (ids >= 0) & torch.isfinite(t)
            taught = there.any(1)
            p = torch.nan_to_num(torch.softmax(t.masked_fill(~there, -math.inf), 1))
            soft = torch.zeros(R, V, **f64)
            r, k = there.nonzero(as_tuple=True)
            soft.index_put_((r, ids[r, k]), p[r, k], accumulate=True)
        counts = labelled | taught
        if not back:
            L = torch.logsumexp(z, 1)
            loss = lw * (hard * (L[:, None] - z)).sum(1) + zw * L ** 2
            o = {}
            if teacher:
                Lt = torch.logsumexp(z / tau, 1)
                entropy = torch.special.xlogy(p, p).sum(1)
                loss = loss + kw * tau ** 2 * (entropy + (soft * (Lt[:, None] - z / tau)).sum(1))
                o = dict(lse_t=Lt * counts, z_top=torch.where(there, z.gather(1, ids.clamp(min=0)), 0.0))
            parts.append(dict(loss=loss * counts, lse=L * counts, **o))
            continue
        lse = s["lse"][m: m + step].double()[:, None]
        q = torch.exp(z - lse)
        d = lw * (q * labelled[:, None] - hard) + 2 * zw * lse * q
        if teacher:
            d = d + kw * tau * (torch.exp(z / tau - s["lse_t"][m: m + step].double()[:, None]) * taught[:, None] - soft)
        d = d * (n["scale"] * s["dloss"][m: m + step].double() * counts)[:, None]
        dW += torch.mm(d.t().contiguous(), h)
        parts.append(dict(dh=torch.mm(d, W)))
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    return out | dict(dW=dW) if back else out
