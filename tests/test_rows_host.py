"""Operators on rows of channels, what needs no GPU: the reference against itself (codes by exhaustion, gradients against
differences), sizes, and what the C ABI refuses before any launch."""
import ctypes

import numpy as np
import pytest

from tests import rows_reference as R
from paper_1901_07988_amd import binding as B


# ---- the reference ------------------------------------------------------------------------------------
@pytest.mark.parametrize("K", [4, 8])
def test_reference_store_is_nearest_and_idempotent(K):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 70)) * np.exp(rng.standard_normal((50, 70)) * 3)
    s = R.pack(x, K)
    v = R.unpack(s, 50, 70, K)
    xb, vb = R.blocked(x), R.blocked(v)
    byte = R.scale_bytes(xb, K).astype(int)[..., None]
    unit = np.ldexp(1.0, byte - 127)
    # no error beyond half the distance of neighbouring codes: unit / 2 (K = 8); a quarter of the power of two below, K = 4
    half = unit / 2 if K == 8 else np.maximum(unit / 4, np.exp2(np.floor(np.log2(np.maximum(np.abs(xb), 1e-300)))) / 4)
    assert (np.abs(xb - vb) <= half * (1 + 1e-12)).all()
    # every value is exact in bf16 (8 bits of significance)
    m, _ = np.frexp(v)
    assert (m * 256 == np.rint(m * 256)).all()
    # a scale one smaller would overflow
    top = np.abs(xb).max(-1, keepdims=True)
    assert (top / unit < (127.5 if K == 8 else 7)).all() and (top / unit * 2 >= (127.5 if K == 8 else 7)).all()


@pytest.mark.parametrize("gate_rows", [0, 1, 2, 5])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("center", [False, True])
def test_reference_step_gradients_are_differences(gate_rows, post, center):
    rng = np.random.default_rng(2)
    M, C, eps, alpha, beta = 5, 7, 1e-3, 0.7, 0.4
    r, b = rng.standard_normal((2, M, C))
    gate = rng.standard_normal((-(-M // gate_rows), C)) if gate_rows else None
    w_post = rng.standard_normal(C) if post else None
    w_pre = rng.standard_normal(C)
    gr, gn = rng.standard_normal((2, M, C))

    def loss(r, b, gate, w_post, w_pre):
        f = R.step_forward(r, b, gate, gate_rows, w_post, w_pre, alpha, beta, eps, center)
        return (gr * f["r"]).sum() + (gn * f["n"]).sum()

    args = [r, b, gate, w_post, w_pre]
    f = R.step_forward(r, b, gate, gate_rows, w_post, w_pre, alpha, beta, eps, center)
    g = R.step_backward(gn, gr, f["y"], f["rstd_b"], f["z"], f["rstd_n"], gate, gate_rows, w_post, w_pre, alpha, beta, center)
    for k, name in enumerate(("dr", "db", "dgate", "dw_post", "dw_pre")):
        if args[k] is None:
            assert name not in g
            continue
        for at in np.ndindex(args[k].shape):
            h = 1e-5
            hi, lo = [[None if a is None else a.copy() for a in args] for _ in range(2)]
            hi[k][at] += h
            lo[k][at] -= h
            d = (loss(*hi) - loss(*lo)) / (2 * h)
            assert abs(d - g[name][at]) < 1e-6 * max(1.0, abs(d)), (name, at)


@pytest.mark.parametrize("kind", [0, 1])
def test_reference_activation_derivative(kind):
    g = np.linspace(-9, 9, 301)
    h = 1e-5
    d = (R.act(g + h, kind)[0] - R.act(g - h, kind)[0]) / (2 * h)
    np.testing.assert_allclose(R.act(g, kind)[1], d, atol=1e-8)


# ---- sizes and refusals -------------------------------------------------------------------------------
def test_store_sizes():
    for M, C in ((1, 1), (1, 32), (3, 33), (128, 4096), (1000, 1111)):
        for K in (4, 8):
            assert B.abl_ckpt_bytes(M, C, K) == R.store_size(M, C, K)
    assert B.abl_ckpt_bytes(0, 64, 8) > 0
    assert B.abl_ckpt_bytes(8192, 4096, 8) * 32 == 8192 * 4096 * 33          # 8.25 bits a value
    # sizes beyond 32 bits
    assert B.abl_ckpt_bytes(1 << 22, 4000, 8) == (1 << 22) * 125 * 33
    for bad in ((-1, 64, 8), (4, 0, 8), (4, 64, 3), (4, 64, 32), (1 << 29, 1, 8), (1 << 20, 1 << 15, 8)):
        assert B.abl_ckpt_bytes(*bad) == 0


P = 4096        # an aligned address that no refused call looks at


def test_pack_and_unpack_refuse():
    ok = dict(dtype=1, x=P, ldx=64, M=4, C=64, K=8, store=P)

    def both(**kw):
        a = {**ok, **kw}
        return {B.lib.abl_ckpt_pack(None, a["dtype"], a["x"], a["ldx"], a["M"], a["C"], a["K"], a["store"]),
                B.lib.abl_ckpt_unpack(None, a["dtype"], a["store"], a["M"], a["C"], a["K"], a["x"], a["ldx"])}

    for kw in (dict(dtype=2), dict(dtype=-1), dict(x=None), dict(x=P + 1), dict(ldx=63), dict(K=0), dict(K=32), dict(store=None),
               dict(store=P + 8), dict(dtype=0, x=P + 2)):
        assert both(**kw) == {B.ABL_ERR_ARG}, kw
    for kw in (dict(M=-1), dict(C=0), dict(M=1 << 29), dict(M=1 << 25, C=1 << 10)):
        assert both(**kw) == {B.ABL_ERR_SHAPE}, kw
    assert both(M=0, x=None, store=None) == {B.ABL_OK}


def step(**kw):
    a = dict(M=4, gate_rows=2, C=64, dtype=1, K=8, flags=0, alpha=1.0, beta=1.0, eps=1e-5)
    a.update(kw)
    return B.abl_resnorm(**a)


def test_resnorm_forward_refuses():
    names = ("r", "b", "gate", "w_post", "w_pre", "r_out", "n", "ckpt_b", "rstd_b", "ckpt_n", "rstd_n")

    def call(s, **kw):
        a = dict.fromkeys(names, P)
        a.update(kw)
        return B.lib.abl_resnorm_forward(None, None if s is None else ctypes.byref(s), *[a[k] for k in names])

    assert call(None) == B.ABL_ERR_ARG
    for kw in (dict(dtype=3), dict(K=5), dict(flags=1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(gate_rows=0)):
        assert call(step(**kw)) == B.ABL_ERR_ARG, kw
    for kw in (dict(M=-1), dict(C=0), dict(C=16385), dict(M=(1 << 25) + 1, C=1)):
        assert call(step(**kw)) == B.ABL_ERR_SHAPE, kw
    for name in ("r", "w_pre", "n", "ckpt_n", "rstd_n", "ckpt_b", "rstd_b"):
        assert call(step(), **{name: None}) == B.ABL_ERR_ARG, name
    for name in names:
        assert call(step(), **{name: P + 1}) == B.ABL_ERR_ARG, name
    assert call(step(), b=None) == B.ABL_ERR_ARG                       # a norm or a gate of nothing
    assert call(step(), b=None, gate=None) == B.ABL_ERR_ARG
    assert call(step(M=0), r=None, n=None) == B.ABL_OK


def test_resnorm_backward_refuses():
    names = ("dn", "dr_out", "gate", "w_post", "w_pre", "ckpt_b", "rstd_b", "ckpt_n", "rstd_n", "scratch", "bytes", "dr", "db",
             "dgate", "dw_post", "dw_pre")

    def call(s, has_b=1, **kw):
        a = dict.fromkeys(names, P)
        a["bytes"] = 1 << 30
        a.update(kw)
        return B.lib.abl_resnorm_backward(None, None if s is None else ctypes.byref(s), has_b, *[a[k] for k in names])

    assert call(None) == B.ABL_ERR_ARG
    for kw in (dict(dtype=3), dict(K=0), dict(K=32), dict(flags=2), dict(gate_rows=0)):
        assert call(step(**kw)) == B.ABL_ERR_ARG, kw
    for kw in (dict(M=-1), dict(C=0), dict(C=16385), dict(M=(1 << 25) + 1, C=1)):
        assert call(step(**kw)) == B.ABL_ERR_SHAPE, kw
    for name in ("dn", "w_pre", "ckpt_b", "rstd_b", "ckpt_n", "rstd_n", "scratch", "dgate", "dw_post", "dw_pre", "gate", "w_post"):
        assert call(step(), **{name: None}) == B.ABL_ERR_ARG, name
    for name in names:
        if name != "bytes":
            assert call(step(), **{name: P + 1}) == B.ABL_ERR_ARG, name
    assert call(step(), has_b=0) == B.ABL_ERR_ARG
    need = B.abl_resnorm_scratch_bytes(4, 64)
    assert need > 0 and call(step(), bytes=need - 1) == B.ABL_ERR_SCRATCH
    assert B.abl_resnorm_scratch_bytes(4, 16385) == 0 and B.abl_resnorm_scratch_bytes(-1, 64) == 0


def test_resnorm_workspace_is_enough_for_every_gate_and_stays_small():
    """The shares that the backward cuts the rows into, as its comment describes them, against the size that is asked for."""
    for C in (64, 1024, 1111, 4096, 8192, 16384):
        for M in (1, 7, 300, 2048, 5000, 16384, 100000):
            assert B.abl_resnorm_scratch_bytes(M, C) <= 256 << 20
            assert B.abl_resnorm_scratch_bytes(M, C) >= 3 * 4 * R.blocks_of(C) * 32


def test_glu_refuses():
    f = ("dtype", "act", "g", "ldg", "u", "ldu", "M", "C", "K", "h", "ldh", "sg", "su")
    b = ("dtype", "act", "dh", "lddh", "sg", "su", "M", "C", "K", "dg", "lddg", "du", "lddu", "sh")
    ok = dict(dtype=1, act=0, M=4, C=64, K=8, ldg=64, ldu=128, ldh=64, lddh=64, lddg=64, lddu=64)
    for names, fn in ((f, B.lib.abl_glu_forward), (b, B.lib.abl_glu_backward)):
        def call(**kw):
            return fn(None, *[{**dict.fromkeys(names, P), **ok, **kw}[k] for k in names])
        for kw in (dict(dtype=7), dict(act=2), dict(act=-1), dict(K=5)):
            assert call(**kw) == B.ABL_ERR_ARG, kw
        for kw in (dict(M=-1), dict(C=0), dict(M=1 << 29)):
            assert call(**kw) == B.ABL_ERR_SHAPE, kw
        for k in names:
            if k.startswith("ld"):
                assert call(**{k: 63}) == B.ABL_ERR_ARG, k
            elif k not in ok:
                assert call(**{k: P + 1}) == B.ABL_ERR_ARG, k
                if k != "sh":
                    assert call(**{k: None}) == B.ABL_ERR_ARG, k
        assert call(M=0) == B.ABL_OK
    assert B.lib.abl_glu_backward(None, *[{**dict.fromkeys(b, P), **ok, "K": 0}[k] for k in b]) == B.ABL_ERR_ARG


def test_wgrad_refuses():
    names = ("dtype", "flags", "store", "M", "Cin", "K", "scale", "dy", "lddy", "Cout", "scratch", "bytes", "dW")
    ok = dict(dtype=1, flags=0, M=40, Cin=64, K=8, lddy=96, Cout=96, bytes=1 << 30)

    def call(**kw):
        return B.lib.abl_ckpt_wgrad(None, *[{**dict.fromkeys(names, P), **ok, **kw}[k] for k in names])

    for kw in (dict(dtype=2), dict(flags=1), dict(flags=64), dict(K=0), dict(lddy=95), dict(store=None), dict(dy=None), dict(dW=None),
               dict(scratch=None), dict(scale=P + 1), dict(dy=P + 1), dict(dW=P + 2), dict(store=P + 4), dict(scratch=P + 8)):
        assert call(**kw) == B.ABL_ERR_ARG, kw
    for kw in (dict(M=-1), dict(Cin=0), dict(Cout=0), dict(Cin=1 << 16, Cout=1 << 15), dict(Cin=(1 << 20) + 1, Cout=1)):
        assert call(**kw) == B.ABL_ERR_SHAPE, kw
    import torch
    for M, ci, co in ((1, 1, 1), (8192, 64, 64), (16384, 4096, 4096)):
        need = B.abl_ckpt_wgrad_scratch_bytes(M, ci, co, torch.bfloat16)
        assert 0 < need <= 256 << 20
        assert call(M=M, Cin=ci, Cout=co, lddy=co, bytes=need - 1) == B.ABL_ERR_SCRATCH
    assert B.abl_ckpt_wgrad_scratch_bytes(4, 64, 64, torch.float16) == 0


def test_wgrad_workspace_stays_small_for_long_batches():
    """Rows beyond what one product's offsets reach are further products: no copies of dW for them."""
    import torch
    for M, ci, co in ((1 << 18, 8192, 32768), (1 << 20, 4096, 8192), (1 << 13, 1 << 20, 2047), (1 << 13, 2047, 1 << 20), (1 << 22, 96, 64)):
        for dtype in (torch.bfloat16, torch.float32):
            assert 0 < B.abl_ckpt_wgrad_scratch_bytes(M, ci, co, dtype) <= 256 << 20


def test_workspaces_of_no_rows_have_a_size():
    """M = 0 is a valid batch: every size is given, and none is that of invalid arguments."""
    import torch
    for C in (1, 64, 513, 1111, 8193, 16384):
        assert 0 < B.abl_resnorm_scratch_bytes(0, C) <= B.abl_resnorm_scratch_bytes(1, C)
        assert B.abl_ckpt_bytes(0, C, 4) == B.abl_ckpt_bytes(0, C, 8) == 128
        for dtype in (torch.bfloat16, torch.float32):
            assert B.abl_ckpt_wgrad_scratch_bytes(0, C, C, dtype) > 0


def test_the_other_operators_do_without_the_compiled_marshalling(tmp_path):
    """_rows.so absent, or built against another torch: everything else is there, and the operators on rows say what is missing."""
    import os
    import shutil
    import subprocess
    import sys
    package = os.path.dirname(B.__file__)
    for bad in (None, b"not a library"):
        there = tmp_path / ("none" if bad is None else "bad")
        shutil.copytree(package, there / "paper_1901_07988_amd", ignore=shutil.ignore_patterns("_rows.so", "csrc", "__pycache__"))
        if bad is not None:
            (there / "paper_1901_07988_amd" / "_rows.so").write_bytes(bad)
        run = subprocess.run([sys.executable, "-c", """
from paper_1901_07988_amd import binding as B, runtime
import os
assert os.getcwd() in os.path.realpath(B.__file__)
assert B.abl_packed_bytes((1, 1, 1, 3, 4, 1, 1, 1, 0), 4) == 128
assert B.abl_ckpt_bytes(4, 64, 8) == 384
for call in (lambda: B.abl_ckpt_pack(None, 8, None), lambda: B.abl_glu_forward(None, None, None, 0)):
    try:
        call()
    except ImportError as e:
        assert "_rows.so" in str(e)
    else:
        raise SystemExit("no error")
"""], cwd=there, capture_output=True, text=True, timeout=300, env={**os.environ, "PYTHONPATH": str(there)})
        assert run.returncode == 0, run.stderr


def shares(M, C, gate_rows):
    """How the backward of the residual step cuts M rows: (rows of a team, teams of a group or 0, blocks that write sums of their own)."""
    pieces = R.blocks_of(C) * 4
    team = next((t for t in (64, 128, 192, 256) if pieces <= t), 512)
    most, block = 128 * 1024 // team, 4 if team == 64 else 1
    rows = -(-M // most)
    if gate_rows and gate_rows <= rows:
        rows, per_group = -(-rows // gate_rows) * gate_rows, 0
        teams = -(-M // rows)
    elif gate_rows:
        group = min(gate_rows, M)
        per_group = -(-(-(-group // rows)) // block) * block
        rows = -(-group // per_group)
        teams = -(-M // group) * per_group
    else:
        per_group, teams = 0, -(-M // rows)
    return rows, per_group, -(-teams // block)


def test_resnorm_workspace_holds_the_sums_of_every_cut():
    """Three planes of a block's sums for every way to cut the rows: no gate, groups below, at and beyond a team's rows, one group of all."""
    rng = np.random.default_rng(0)
    cuts = set()
    for C in (1, 40, 512, 513, 1000, 1111, 1536, 1537, 2048, 2100, 4096, 4104, 8192, 8193, 16384):
        for M in [1, 2, 7, 300, 2047, 2048, 2049, 5000, 16384, 70000, 100001, 1 << 22] + [int(2 ** rng.uniform(0, 22)) for _ in range(40)]:
            if M * R.blocks_of(C) >= 1 << 29:      # (refused)
                continue
            have = B.abl_resnorm_scratch_bytes(M, C)
            rows = shares(M, C, 0)[0]
            for g in {0, 1, 2, 3, rows - 1, rows, rows + 1, 2 * rows, 2 * rows + 1, M // 3, M // 2, M - 1, M, M + 1, 1 << 40} | {
                    int(2 ** rng.uniform(0, 22)) for _ in range(4)}:
                if g < 0:
                    continue
                team_rows, per_group, blocks = shares(M, C, g)
                cuts.add((g > 0, per_group > 1, team_rows > 1))
                assert blocks * 3 * R.blocks_of(C) * 32 * 4 <= have, (M, C, g)
    assert len(cuts) >= 6, cuts
