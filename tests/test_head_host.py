"""Losses over a vocabulary, what needs no GPU: the reference against itself (gradients against differences), sizes, and what the C ABI
refuses before any launch."""
import ctypes
import math
import random

import pytest
import torch

from tests import head_reference as R
from paper_1901_07988_amd import binding as B
from paper_1901_07988_amd import token_head as H


# ---- the reference ------------------------------------------------------------------------------------
@pytest.mark.parametrize("teacher", [False, True])
@pytest.mark.parametrize("tau,smoothing,z_weight", [(1.0, 0.0, 0.0), (1.0, 0.2, 0.01), (2.5, 0.1, 0.003)])
def test_reference_gradients_are_differences(teacher, tau, smoothing, z_weight):
    gen = torch.Generator().manual_seed(3)
    M, C, V, T = 5, 4, 7, 3
    h, W = torch.randn(M, C, generator=gen, dtype=R.F64), torch.randn(V, C, generator=gen, dtype=R.F64)
    labels = torch.tensor([2, -1, 0, 6, -5])
    n = R.Settings(scale=1.3, smoothing=smoothing, z_weight=z_weight, temperature=tau, label_weight=0.7, teacher_weight=0.9 if teacher else 0.0)
    ids = torch.tensor([[1, 1, 2], [0, -1, 4], [-1, -1, -1], [3, 5, 6], [-1, -2, -1]]) if teacher else None
    t = torch.tensor([[0.3, 1.0, -0.5], [1.0, 9.0, 0.0], [1.0, 2.0, 3.0], [0.1, -float("inf"), 2.0], [0.0, 0.0, 0.0]]) if teacher else None
    w = torch.randn(M, generator=gen, dtype=R.F64)

    def loss(h, W):
        return (w * R.forward(h, W, labels, n, ids, t)["loss"]).sum()

    f = R.forward(h, W, labels, n, ids, t)
    assert f["loss"][4] == 0 and f["lse"][4] == 0
    g = R.backward(h, W, labels, f["lse"], w, n, torch.float32, torch.float32, ids=ids, t=t, lse_t=f.get("lse_t"))
    for name, x in (("dh", h), ("dW", W)):
        for i in range(x.shape[0]):
            for j in range(x.shape[1]):
                hi, lo = x.clone(), x.clone()
                hi[i, j] += 1e-6
                lo[i, j] -= 1e-6
                d = (loss(hi, W) - loss(lo, W) if name == "dh" else loss(h, hi) - loss(h, lo)) / 2e-6
                assert abs(d - g[name][i, j]) < 1e-7 * max(1.0, abs(float(d))), (name, i, j)


def test_reference_losses_are_torchs():
    gen = torch.Generator().manual_seed(4)
    h, W = torch.randn(6, 5, generator=gen, dtype=R.F64), torch.randn(9, 5, generator=gen, dtype=R.F64)
    labels = torch.tensor([0, 8, 3, -100, 2, 2])
    z = h @ W.t()
    f = R.forward(h, W, labels, R.Settings(smoothing=0.1))
    want = torch.nn.functional.cross_entropy(z, labels, reduction="none", label_smoothing=0.1)
    torch.testing.assert_close(f["loss"], want)
    # every token an entry: the divergence of two softmaxes
    t = torch.randn(6, 9, generator=gen)
    ids = torch.stack([torch.randperm(9, generator=gen) for _ in range(6)])
    n = R.Settings(temperature=2.0, label_weight=0.0, teacher_weight=1.0)
    f = R.forward(h, W, None, n, ids, t)
    dense = torch.zeros(6, 9, dtype=R.F64).scatter_(1, ids, t.double())
    want = 4 * torch.nn.functional.kl_div(torch.log_softmax(z / 2, 1), torch.softmax(dense / 2, 1), reduction="none").sum(1)
    torch.testing.assert_close(f["loss"], want)


# ---- sizes --------------------------------------------------------------------------------------------
def test_scratch_sizes():
    size = B.abl_head_scratch_bytes
    f32, bf16 = torch.float32, torch.bfloat16
    assert size(1, 1, 1, f32) > 0 and size(0, 1, 1, bf16, backward=True) > 0
    # the logits of this call would be 2 GB; what it takes beside a copy of the rows stays below 512 MB (rows: 64 MB, their gradient's sums: 128 MB)
    assert size(8192, 4096, 65536, bf16, backward=True) < (512 + 192) << 20
    assert size(8192, 4096, 65536, bf16) < (192 + 64) << 20
    assert size(1 << 20, 1024, 1 << 17, bf16, backward=True) > 1 << 32
    for kw in (dict(M=-1), dict(C=0), dict(V=0), dict(M=(1 << 23) + 1), dict(C=(1 << 16) + 1), dict(V=(1 << 26) + 1), dict(M=1 << 23, V=1 << 22),
               dict(T=1025), dict(T=-1), dict(dtype=torch.float16), dict(dw_dtype=torch.float16, backward=True),
               dict(dtype=f32, dw_dtype=bf16, backward=True), dict(flags=B.ABL_ACCUM_DW), dict(flags=1)):
        assert size(**{**dict(M=4, C=8, V=16, dtype=bf16), **kw}) == 0, kw
    assert size(4, 8, 16, bf16, flags=B.ABL_ACCUM_DW | B.ABL_MATH_BF16, backward=True) > 0
    assert B.lib.abl_head_scratch_bytes(None, 0) == 0


def layouts(p):
    """(size of a workspace as it is given, sizes of what calls lay out there: the table where it is, copied), forward and backward."""
    lay = B.lib.abl_head_layout_bytes
    lay.restype, lay.argtypes = ctypes.c_size_t, [ctypes.POINTER(B.abl_head), ctypes.c_int, ctypes.c_int]
    r = ctypes.byref(p)
    return [(B.lib.abl_head_scratch_bytes(r, b), lay(r, b, 0), lay(r, b, 1)) for b in (0, 1)]


def test_no_call_lays_out_more_than_its_workspace():
    """The launchers compare a call's own layout with what they are given (ABL_ERR_SCRATCH); a workspace of the size that is asked for is enough."""
    rng = random.Random(11)

    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    sizes = [(M, C, V, T, t) for M in (0, 1, 16, 17, 64, 65, 256, 257, 1024, 1025) for C in (1, 64, 65, 4096, 1 << 16) for V in (1, 255, 257, 32000, 1 << 26)
             for T in (0, 1024) for t in range(4)]
    sizes += [(1 << 23, 1 << 16, 1 << 21, T, t) for T in (0, 7) for t in range(4)]
    sizes += [(size(1, 8192) if i % 8 else size(1, 1 << 23), size(1, 8192), size(1, 131072), rng.choice([0, 0, 1, 25]), rng.randrange(4)) for i in range(60000)]
    types = [(B.ABL_BF16, B.ABL_BF16, 0), (B.ABL_BF16, B.ABL_F32, 0), (B.ABL_F32, B.ABL_F32, 0), (B.ABL_F32, B.ABL_F32, B.ABL_MATH_BF16)]
    for M, C, V, T, t in sizes:
        if M * V > 1 << 44:
            continue
        d, w, flags = types[t]
        for given, in_place, copied in layouts(B.abl_head(M=M, C=C, V=V, T=T, dtype=d, dw_dtype=w, flags=flags, scale=1.0, temperature=1.0)):
            assert given > 0 and 0 < in_place <= given and 0 < copied <= given, (M, C, V, T, d, w, flags)


@pytest.mark.parametrize("type,M,C,V,T,need", [(torch.float32, 512, 4096, 32000, 0, 110573824), (torch.float32, 256, 4096, 32768, 0, 91430144),
                                               (torch.float32, 1024, 4096, 50257, 0, 123695360), (torch.float32, 128, 4096, 32000, 0, 91430144),
                                               (torch.bfloat16, 100, 8192, 20000, 0, 105684224), (torch.float32, 512, 2882, 15078, 25, 98600000)])
def test_room_for_logits_in_shares_of_a_copied_table(type, M, C, V, T, need):
    """A table that is copied a piece at a time, whose logits are few enough to be made in shares, where the whole vocabulary's are not: copies of the rows and of a
    piece of the table, and eight slabs of its logits, all at once."""
    assert B.abl_head_scratch_bytes(M, C, V, type, T=T) >= need


# ---- refusals -----------------------------------------------------------------------------------------
P = 4096        # an aligned address that no refused call looks at
CALLS = {
    "abl_xent_forward": ("h", "ldh", "W", "ldw", "labels", "scratch", "bytes", "loss", "lse"),
    "abl_xent_backward": ("h", "ldh", "W", "ldw", "labels", "lse", "dloss", "scratch", "bytes", "dh", "lddh", "dW"),
    "abl_distill_forward": ("h", "ldh", "W", "ldw", "labels", "top_ids", "top_logits", "scratch", "bytes", "loss", "lse", "lse_t", "z_top"),
    "abl_distill_backward": ("h", "ldh", "W", "ldw", "labels", "top_ids", "top_logits", "lse", "lse_t", "z_top", "dloss", "scratch", "bytes", "dh",
                             "lddh", "dW"),
}
HEAD = dict(M=4, C=8, V=16, T=3, dtype=B.ABL_BF16, dw_dtype=B.ABL_BF16, flags=0, scale=1.0, smoothing=0.1, z_weight=0.0, temperature=2.0,
            label_weight=1.0, teacher_weight=1.0)


def call(name, head={}, **kw):
    p = None if head is None else ctypes.byref(B.abl_head(**{**HEAD, **head}))
    a = {**dict.fromkeys(CALLS[name], P), "ldh": 8, "ldw": 8, "lddh": 8, "bytes": 1 << 40, **kw}
    return getattr(B.lib, name)(None, p, *[a[k] for k in CALLS[name]])


@pytest.mark.parametrize("name", list(CALLS))
def test_calls_refuse(name):
    nan, inf = float("nan"), float("inf")
    back, teacher = name.endswith("backward"), "distill" in name
    assert call(name, None) == B.ABL_ERR_ARG
    wrong = [dict(dtype=2), dict(dtype=-1), dict(flags=1), dict(flags=B.ABL_NORM_CENTER), dict(scale=nan), dict(scale=inf), dict(smoothing=1.0),
             dict(smoothing=-0.1), dict(smoothing=nan), dict(z_weight=nan)]
    if back:
        wrong += [dict(dw_dtype=2), dict(dtype=B.ABL_F32, dw_dtype=B.ABL_BF16)]
    else:
        wrong += [dict(flags=B.ABL_ACCUM_DW)]
    if teacher:
        wrong += [dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=nan), dict(temperature=inf), dict(temperature=1e-39),
                  dict(label_weight=nan), dict(teacher_weight=inf)]
    for head in wrong:
        assert call(name, head) == B.ABL_ERR_ARG, head
    sizes = [dict(M=-1), dict(M=(1 << 23) + 1), dict(C=0), dict(C=(1 << 16) + 1), dict(V=0), dict(V=(1 << 26) + 1), dict(M=1 << 23, V=1 << 22)]
    for head in sizes + ([dict(T=0), dict(T=-1), dict(T=1025)] if teacher else []):
        assert call(name, head) == B.ABL_ERR_SHAPE, head
    may_be_null = {"dh", "dW"} | ({"labels"} if teacher else set())
    for k in CALLS[name]:
        if k in ("ldh", "ldw", "lddh"):
            assert call(name, **{k: 7}) == B.ABL_ERR_ARG, k
        elif k != "bytes":
            assert call(name, **{k: P + 1}) == B.ABL_ERR_ARG, k
            if k not in may_be_null:
                assert call(name, **{k: None}) == B.ABL_ERR_ARG, k
    assert call(name, scratch=P + 8) == B.ABL_ERR_ARG
    if back:
        assert call(name, dh=None, dW=None) == B.ABL_ERR_ARG
        assert call(name, dict(dw_dtype=B.ABL_F32), dW=P + 2) == B.ABL_ERR_ARG
    if teacher:
        assert call(name, dict(z_weight=0.1), labels=None, lse=None) == B.ABL_ERR_ARG
    need = B.lib.abl_head_scratch_bytes(ctypes.byref(B.abl_head(**{**HEAD, "T": 3 if teacher else 0})), 1 if back else 0)
    assert need > 0 and call(name, bytes=need - 1) == B.ABL_ERR_SCRATCH
    if not back:
        assert call(name, dict(M=0), h=None, labels=None, loss=None) == B.ABL_OK
    else:
        assert call(name, dict(M=0), h=None, dW=None) == B.ABL_OK


def test_calls_refuse_tensors_of_the_cpu():
    x = torch.zeros(4, 8)
    with pytest.raises(AssertionError):
        B.abl_xent_forward(x, x, torch.zeros(4, dtype=torch.int64), None, None, None)


def test_a_head_of_labels_alone_refuses_weights():
    """They would not be looked at: a loss half as large was asked for and not given."""
    for how in (dict(label_weight=0.5), dict(temperature=2.0), dict(teacher_weight=0.0)):
        with pytest.raises(AssertionError):
            H.VocabularyHead(torch.zeros(4, 8), 2, **how)
