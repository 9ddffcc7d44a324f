"""Operators on rows of channels on the GPU against the definitions in 64 bits (rows_reference.py).

Tolerances, u = 2^-24.  Stores of given tensors, and everything read from a store, are exact: bytes are compared.
Element-wise fp32 results of a few operations (gated unit) are held to 32 u of the result's terms: exponential, quotient and four
products stay within 16 u at these magnitudes.  Where a sum over a row goes in (norms), its error with up to 64 terms in turn per
thread and a tree over threads is below 80 u of the sum of magnitudes, so results are held to 2^-16 of the terms'
magnitude.  A sum over M rows is in turn over a share and over the shares: M u of the sum of magnitudes bounds it, and
products of matrices likewise.  bf16 results add half a unit in the last place, 2^-8 of the result (eight bits of significance).  The store of a computed tensor
may differ by one code where the value lies within that error of the middle of two codes.
"""
import numpy as np
import pytest
import torch

from paper_1901_07988_amd import binding as B
from paper_1901_07988_amd import runtime as G
from tests import rows_reference as R

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
U = 2.0 ** -24


def dev(a, dtype):
    return torch.from_numpy(np.array(a)).to("cuda").to(dtype).contiguous()


def f64(t):
    return t.detach().double().cpu().numpy()


def rounding(dtype):
    return 0.0 if dtype == torch.float32 else 2.0 ** -8


def hold(got, want, magnitude, terms, dtype, what):
    """|got - want| <= terms magnitude + rounding |want|, with NaN where it is expected."""
    got = f64(got)
    assert got.shape == want.shape, what
    assert (np.isnan(got) == np.isnan(want)).all(), what
    bound = terms * np.broadcast_to(magnitude, want.shape) + (rounding(dtype) * 1.01) * np.abs(want) + 1e-37
    off = np.abs(got - want) - bound
    assert not (off > 0).any(), (what, float(np.nanmax(off / bound)))


def store(M, C, K):
    return torch.full((B.abl_ckpt_bytes(M, C, K),), 0xEE, dtype=torch.uint8, device="cuda")


def tensor(*shape, dtype=torch.float32):
    return torch.full(shape, 7.0, dtype=dtype, device="cuda")


def heavy(rng, M, C):
    return rng.standard_normal((M, C)) * np.exp(rng.standard_normal(C) * 0.7)


SHAPES = [(1, 1), (1, 31), (2, 32), (3, 33), (5, 100), (64, 256), (7, 1111), (1, 8192), (300, 40)]


# ---- block stores -------------------------------------------------------------------------------------
@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C", SHAPES)
def test_pack_writes_the_bytes_of_the_definition(M, C, dtype, K):
    rng = np.random.default_rng(M * 1000 + C)
    x = dev(heavy(rng, M, C), dtype)
    s = store(M, C, K)
    B.abl_ckpt_pack(x, K, s)
    np.testing.assert_array_equal(s.cpu().numpy(), R.pack(f64(x), K))
    for out in TYPES:                                              # every value is exact in both types
        v = tensor(M, C, dtype=out)
        B.abl_ckpt_unpack(s, K, v)
        np.testing.assert_array_equal(f64(v), R.unpack(s.cpu().numpy(), M, C, K))


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
def test_pack_at_ties_limits_and_extreme_sizes(dtype, K):
    """Rows of quarter codes (every tie between two codes), of maxima around the value that takes the next scale, of zeros, tiny and huge
    values; with both signs."""
    limit = 127.5 if K == 8 else 7.0
    rows = []
    grid = np.arange(0, 512) / 4 if K == 8 else np.arange(0, 28) / 4
    grid = np.resize(grid, 512)
    for e in (0, -7, 9, -118, 100):
        rows += [np.ldexp(grid, e), -np.ldexp(grid, e)]
    for top in (limit, np.nextafter(np.float32(limit), np.float32(0)), np.nextafter(np.float32(limit), np.float32(1e9)), limit * 2, 126.5, 6.0):
        row = np.full(512, 0.3)
        row[5::32] = top
        rows.append(row)
    rows += [np.zeros(512), np.full(512, -0.0), np.full(512, 1e-40), np.full(512, 2.0 ** -126), np.full(512, 3.3e38), np.full(512, -3.3e38)]
    x = dev(np.stack(rows).astype(np.float32), dtype)
    M, C = x.shape
    s = store(M, C, K)
    B.abl_ckpt_pack(x, K, s)
    want = R.pack(f64(x), K)
    got = s.cpu().numpy()
    n = M * (C // 32) * 4 * K
    np.testing.assert_array_equal(got[n:], want[n:])
    np.testing.assert_array_equal(R.unpack(got, M, C, K), R.unpack(want, M, C, K))   # (a code of zero may carry either sign)


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_a_block_with_an_infinity_or_nan_reads_as_nan_and_no_other(bad, dtype, K):
    x = dev(np.random.default_rng(3).standard_normal((4, 100)), dtype)
    x[1, 40] = bad
    x[3, 99] = bad
    s = store(4, 100, K)
    B.abl_ckpt_pack(x, K, s)
    np.testing.assert_array_equal(s.cpu().numpy(), R.pack(f64(x), K))
    v = tensor(4, 100)
    B.abl_ckpt_unpack(s, K, v)
    nan = torch.isnan(v).cpu().numpy()
    want = np.zeros((4, 100), bool)
    want[1, 32:64] = want[3, 96:] = True
    np.testing.assert_array_equal(nan, want)


@pytest.mark.parametrize("K", [4, 8])
def test_unpack_of_every_code_and_scale(K):
    codes = np.arange(256, dtype=np.uint8)
    B_ = 8 if K == 8 else 16
    scales = [8, 9, 60, 126, 127, 128, 200, 248, 255]
    M = len(scales)
    raw = np.zeros(R.store_size(M, 32 * B_, K), np.uint8)
    n = M * B_ * 4 * K
    raw[:n] = np.resize(codes, n)
    raw[n: n + M * B_] = np.repeat(scales, B_)
    v = tensor(M, 32 * B_)
    B.abl_ckpt_unpack(torch.from_numpy(raw).cuda(), K, v)
    np.testing.assert_array_equal(f64(v), R.unpack(raw, M, 32 * B_, K).astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first,C,wide", [(0, 64, 72), (3, 61, 77), (1, 96, 100), (8, 8, 16)])
def test_slices_are_read_and_written_in_place(first, C, wide, dtype, K):
    M = 9
    big = dev(np.random.default_rng(4).standard_normal((M, wide)), dtype)
    x = big[:, first: first + C]
    s = store(M, C, K)
    B.abl_ckpt_pack(x, K, s)
    np.testing.assert_array_equal(s.cpu().numpy(), R.pack(f64(x), K))
    out = tensor(M, wide, dtype=dtype)
    B.abl_ckpt_unpack(s, K, out[:, first: first + C])
    want = np.full((M, wide), 7.0)
    want[:, first: first + C] = R.unpack(s.cpu().numpy(), M, C, K)
    np.testing.assert_array_equal(f64(out), want)


def test_stores_beyond_32_bits_of_offsets():
    """2^31 elements and more: the last rows, and what lies around 2^31 and 2^32 bytes."""
    M, C, K = (1 << 21) + 3, 1056, 8
    x = torch.zeros(M, C, dtype=torch.bfloat16, device="cuda")
    at = [0, 1, (1 << 31) // C - 1, (1 << 31) // C, (1 << 31) // C + 1, (1 << 30) // C, M - 2, M - 1]
    rows = dev(np.random.default_rng(5).standard_normal((len(at), C)), torch.bfloat16)
    x[at] = rows
    s = store(M, C, K)
    B.abl_ckpt_pack(x, K, s)
    x.fill_(3.0)
    B.abl_ckpt_unpack(s, K, x)
    small = R.pack(f64(rows), K)
    np.testing.assert_array_equal(f64(x[at]), R.unpack(small, len(at), C, K))
    left = torch.ones(M, dtype=torch.bool, device="cuda")
    left[at] = False
    assert x.abs().amax(1)[left].max().item() == 0.0


# ---- residual step ------------------------------------------------------------------------------------
def codes_may_differ(got, exact, M, C, K, what):
    """The store of a computed tensor against that of its values in 64 bits.  A block has the scale of the definition, or the other one where
    its maximum lies within 2^-16 of the value that separates the two; given the scale, a code is the nearest, or the neighbouring one where
    the value lies within 2^-16 of its row's terms of the middle between the two."""
    raw = got.cpu().numpy()
    n = M * R.blocks_of(C) * 4 * K
    byte = raw[n: n + M * R.blocks_of(C)].reshape(M, -1)
    want = R.scale_bytes(R.blocked(exact), K)
    top = np.abs(R.blocked(exact)).max(-1)
    limit = 127.5 if K == 8 else 7.0
    edge = np.ldexp(limit, np.minimum(byte, want).astype(int) - 127)
    ok = (byte == want) | ((np.abs(byte.astype(int) - want) == 1) & (np.abs(top - edge) <= 2.0 ** -16 * edge))
    assert ok.all(), what
    got, want = R.unpack(raw, M, C, K), R.unpack(R.pack(exact, K, byte), M, C, K)
    same = got == want
    middle = (got + want) / 2
    room = 2.0 ** -16 * (np.abs(exact) + np.sqrt((exact ** 2).mean(1, keepdims=True)))
    assert (np.abs(exact - middle)[~same] <= np.broadcast_to(room, exact.shape)[~same]).all(), what
    # (not rare for h: where act(g) is g but for 1e-9 of it, h is a product of two codes, and such products often are middles)
    assert (~same).mean() < 0.02 + 2 / same.size, what


def draw_step(rng, M, C, rows, post, has_b, dtype):
    d = dict(r=dev(heavy(rng, M, C), dtype), b=dev(heavy(rng, M, C), dtype) if has_b else None,
             gate=dev(rng.standard_normal((-(-M // rows), C)) * 0.3 + 0.5, dtype) if rows and has_b else None,
             w_post=dev(rng.standard_normal(C) * 0.2 + 1, dtype) if post and has_b else None,
             w_pre=dev(rng.standard_normal(C) * 0.2 + 1, dtype))
    return d, {k: None if v is None else f64(v) for k, v in d.items()}


STEPS = [  # M, C, gate_rows, post, center, K, has_b
    (1, 1, 0, False, False, 8, True),
    (1, 7, 1, True, False, 4, True),
    (2, 32, 2, True, True, 8, True),
    (3, 100, 2, False, False, 8, True),
    (5, 512, 0, True, False, 8, True),
    (6, 520, 1, True, True, 4, True),
    (9, 1111, 4, True, False, 8, True),
    (33, 1024, 33, True, False, 8, True),
    (17, 2048, 5, False, True, 8, True),
    (4, 4096, 0, False, False, 8, True),
    (3, 4104, 1, True, False, 8, True),
    (3, 8192, 2, True, True, 8, True),
    (2, 8200, 0, True, False, 4, True),
    (2, 16384, 1, True, True, 8, True),
    (5, 300, 0, False, False, 8, False),
    (5, 300, 0, False, True, 4, False),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C,rows,post,center,K,has_b", STEPS)
def test_step_forward(M, C, rows, post, center, K, has_b, dtype):
    alpha, beta, eps = 0.75, 0.5, 1e-5
    d, h = draw_step(np.random.default_rng(C), M, C, rows, post, has_b, dtype)
    want = R.step_forward(h["r"], h["b"], h["gate"], rows, h["w_post"], h["w_pre"], alpha, beta, eps, center)
    keep_b = has_b and (post or rows)
    flags = B.ABL_NORM_CENTER if center else 0
    out = {}
    for k in (0, K):
        r_out, n = tensor(M, C, dtype=dtype), tensor(M, C, dtype=dtype)
        sn, sb = store(M, C, K), store(M, C, K) if keep_b else None
        rn, rb = tensor(M), tensor(M)
        B.abl_resnorm_forward(d["r"], d["b"], d["gate"], rows, d["w_post"], d["w_pre"], r_out, n, k, sb, rb if post else None, sn, rn,
                              alpha, beta, eps, flags)
        out[k] = (r_out, n)
    assert torch.equal(out[0][0], out[K][0]) and torch.equal(out[0][1], out[K][1])
    size_r = np.abs(alpha * h["r"])
    if has_b:
        p = want["y"] * (h["w_post"] if post else 1) * (R.gate_rows_of(h["gate"], rows, M) if rows else 1)
        size_r = size_r + np.abs(beta * p) + (beta * np.abs(h["b"]).max(1, keepdims=True) * want["rstd_b"][:, None] if post and center else 0)
    hold(r_out, want["r"], size_r, 2.0 ** -16, dtype, "r")
    scale = want["rstd_n"][:, None] * (size_r + (size_r.max(1, keepdims=True) if center else 0))
    hold(n, want["n"], (np.abs(want["z"]) + scale) * np.abs(h["w_pre"]), 2.0 ** -16, dtype, "n")
    hold(rn, want["rstd_n"], want["rstd_n"], 2.0 ** -16, torch.float32, "rstd_n")
    codes_may_differ(sn, want["z"], M, C, K, "ckpt_n")
    if post and has_b:
        hold(rb, want["rstd_b"], want["rstd_b"], 2.0 ** -16, torch.float32, "rstd_b")
        codes_may_differ(sb, want["y"], M, C, K, "ckpt_b")
    elif keep_b:
        np.testing.assert_array_equal(sb.cpu().numpy(), R.pack(h["b"], K))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C,rows,post,center,K,has_b", STEPS + [
    (2100, 64, 0, True, False, 8, True),      # more rows than teams, every way to cut the groups of a gate
    (5000, 40, 1, True, False, 4, True),
    (5000, 40, 3, False, False, 8, True),
    (4999, 40, 700, True, True, 8, True),
    (4999, 40, 4999, True, False, 8, True),
    (2500, 2100, 1300, True, False, 8, True),
    (2500, 2100, 2, True, False, 8, True),
])
def test_step_backward(M, C, rows, post, center, K, has_b, dtype):
    alpha, beta = 0.75, 0.5
    rng = np.random.default_rng(C + 1)
    d, h = draw_step(rng, M, C, rows, post, has_b, dtype)
    dn, dr_out = (dev(rng.standard_normal((M, C)) * 0.02, dtype) for _ in range(2))
    rn, rb = (dev(np.exp(rng.standard_normal(M) * 0.3), torch.float32) for _ in range(2))
    keep_b = has_b and (post or rows)
    sn, sb = (R.pack(rng.standard_normal((M, C)), K) for _ in range(2))
    z, y = R.unpack(sn, M, C, K), R.unpack(sb, M, C, K)
    scratch = torch.full((B.abl_resnorm_scratch_bytes(M, C),), 0xFF, dtype=torch.uint8, device="cuda")
    for with_dr in ((True, False) if M < 100 else (True,)):
        want = R.step_backward(f64(dn), f64(dr_out) if with_dr else None, y, f64(rb), z, f64(rn), h["gate"], rows, h["w_post"], h["w_pre"],
                               alpha, beta, center, has_b)
        dr, db = tensor(M, C, dtype=dtype), tensor(M, C, dtype=dtype) if has_b else None
        f32 = {k: tensor(*v.shape) for k, v in want.items() if k not in ("dr", "db")}
        B.abl_resnorm_backward(dn, dr_out if with_dr else None, d["gate"], rows, d["w_post"], d["w_pre"], K,
                               torch.from_numpy(sb).cuda() if keep_b else None, rb if post and has_b else None, torch.from_numpy(sn).cuda(),
                               rn, scratch, dr, db, f32.get("dgate"), f32.get("dw_post"), f32["dw_pre"], alpha, beta,
                               B.ABL_NORM_CENTER if center else 0, has_b)
        # magnitudes of the terms
        v = np.abs(f64(dn) * h["w_pre"])
        D = f64(rn)[:, None] * (v + np.abs(z) * (v * np.abs(z)).mean(1, keepdims=True) + v.mean(1, keepdims=True)) + np.abs(f64(dr_out))
        hold(dr, want["dr"], alpha * D, 2.0 ** -16, dtype, "dr")
        hold(f32["dw_pre"], want["dw_pre"], np.abs(f64(dn) * z).sum(0), U * M + 8 * U, torch.float32, "dw_pre")
        if not has_b:
            continue
        e = beta * D * (np.abs(R.gate_rows_of(h["gate"], rows, M)) if rows else 1)
        terms = 2.0 ** -16 + U * M
        if rows:
            t = beta * D * np.abs(y * (h["w_post"] if post else 1))
            G_ = -(-M // rows)
            hold(f32["dgate"], want["dgate"], np.stack([t[g * rows: (g + 1) * rows].sum(0) for g in range(G_)]), terms, torch.float32, "dgate")
        if post:
            hold(f32["dw_post"], want["dw_post"], (e * np.abs(y)).sum(0), terms, torch.float32, "dw_post")
            v = e * np.abs(h["w_post"])
            e = f64(rb)[:, None] * (v + np.abs(y) * (v * np.abs(y)).mean(1, keepdims=True) + v.mean(1, keepdims=True))
        hold(db, want["db"], e, 2.0 ** -16, dtype, "db")


@pytest.mark.parametrize("dtype", TYPES)
def test_step_in_place_and_repeated_is_the_same_bit_for_bit(dtype):
    """Outputs over inputs, as a training program keeps its two streams; and every call gives the same bits again."""
    M, C, K, rows = 700, 1000, 8, 300
    rng = np.random.default_rng(9)
    d, _ = draw_step(rng, M, C, rows, True, True, dtype)
    ref = None
    for alias in (False, True, True):
        r, b = d["r"].clone(), d["b"].clone()
        r_out, n = (r, b) if alias else (tensor(M, C, dtype=dtype), tensor(M, C, dtype=dtype))
        sn, sb, rn, rb = store(M, C, K), store(M, C, K), tensor(M), tensor(M)
        B.abl_resnorm_forward(r, b, d["gate"], rows, d["w_post"], d["w_pre"], r_out, n, K, sb, rb, sn, rn)
        dn, dres = d["r"].clone() * 0.1, d["b"].clone() * 0.1
        dr, db = (dres, dn) if alias else (tensor(M, C, dtype=dtype), tensor(M, C, dtype=dtype))
        g, wp, wq = tensor(-(-M // rows), C), tensor(C), tensor(C)
        ws = torch.empty(B.abl_resnorm_scratch_bytes(M, C), dtype=torch.uint8, device="cuda")
        B.abl_resnorm_backward(dn, dres, d["gate"], rows, d["w_post"], d["w_pre"], K, sb, rb, sn, rn, ws, dr, db, g, wp, wq)
        got = [r_out, n, sn, sb, rn, rb, dr, db, g, wp, wq]
        if ref is None:
            ref = [t.clone() for t in got]
        for a, c in zip(ref, got):
            assert torch.equal(a, c)


def test_step_of_no_rows_and_rows_of_zeros():
    C = 96
    f = dict(dtype=torch.bfloat16, device="cuda")
    w = torch.ones(C, **f)
    none = torch.empty(0, C, **f)
    wp, wq = tensor(C), tensor(C)
    B.abl_resnorm_forward(none, none, None, 0, w, w, none, none)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    one = store(1, C, 8)
    B.abl_resnorm_backward(none, none, None, 0, w, w, 8, one, wp, one, wp, ws, none, none, None, wp, wq)
    assert wp.abs().max().item() == 0 and wq.abs().max().item() == 0
    z = torch.zeros(3, C, **f)
    n, r, rn, rb = z + 1, z + 1, tensor(3), tensor(3)
    sb, sn = store(3, C, 4), store(3, C, 4)
    B.abl_resnorm_forward(z, z, None, 0, w, w, r, n, 4, sb, rb, sn, rn, eps=1e-4)
    assert n.abs().max().item() == 0 and r.abs().max().item() == 0
    np.testing.assert_allclose(rn.cpu().numpy(), 100.0, rtol=1e-6)


def test_step_keeps_a_nan_row_to_itself():
    M, C = 8, 256
    x = torch.randn(M, C, device="cuda")
    b = torch.randn(M, C, device="cuda")
    b[3, 17] = float("nan")
    x[5, 0] = float("inf")
    w = torch.ones(C, device="cuda")
    n, sn, sb, rn, rb = tensor(M, C), store(M, C, 8), store(M, C, 8), tensor(M), tensor(M)
    B.abl_resnorm_forward(x, b, None, 0, w, w, None, n, 8, sb, rb, sn, rn)
    bad = torch.isnan(n).any(1).cpu().numpy()
    np.testing.assert_array_equal(bad, np.isin(np.arange(M), [3, 5]))
    v = tensor(M, C)
    B.abl_ckpt_unpack(sn, 8, v)
    assert torch.isnan(v[3]).all() and torch.isnan(v[5, :32]).all() and not torch.isnan(v[[0, 1, 2, 4, 6, 7]]).any()


# ---- gated unit ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("joint", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C", SHAPES)
def test_gated_unit(M, C, dtype, joint, kind):
    rng = np.random.default_rng(M + C)

    def pair():
        t = tensor(M, 2 * C, dtype=dtype) if joint else None
        return (t[:, :C], t[:, C:]) if joint else (tensor(M, C, dtype=dtype), tensor(M, C, dtype=dtype))

    g, u = pair()
    g.copy_(dev(heavy(rng, M, C) * 2, dtype))
    u.copy_(dev(heavy(rng, M, C), dtype))
    a, _ = R.act(f64(g), kind)
    for K in (0, 4, 8):
        h = tensor(M, C, dtype=dtype)
        sg, su = (store(M, C, K), store(M, C, K)) if K else (None, None)
        B.abl_glu_forward(g, u, h, kind, K, sg, su)
        hold(h, a * f64(u), np.abs(f64(g) * f64(u)), 32 * U, dtype, "h")
        if not K:
            continue
        np.testing.assert_array_equal(sg.cpu().numpy(), R.pack(f64(g), K))
        np.testing.assert_array_equal(su.cpu().numpy(), R.pack(f64(u), K))
        gq, uq = R.unpack(sg.cpu().numpy(), M, C, K), R.unpack(su.cpu().numpy(), M, C, K)
        aq, dq = R.act(gq, kind)
        dh = dev(rng.standard_normal((M, C)) * 0.02, dtype)
        for want_h in (True, False):
            dg, du = pair()
            sh = store(M, C, 8) if want_h else None
            B.abl_glu_backward(dh, sg, su, K, dg, du, kind, sh)
            # act' = s + g s (1 - s) q', q' <= 1.6 + 0.22 g^2, where the product is large s (1 - s) is small: 40 bounds the factor
            hold(dg, f64(dh) * uq * dq, np.abs(f64(dh) * uq) * 40, 32 * U, dtype, "dg")
            hold(du, f64(dh) * aq, np.abs(f64(dh) * gq), 32 * U, dtype, "du")
            if want_h:
                codes_may_differ(sh, aq * uq, M, C, 8, "ckpt_h")


@pytest.mark.parametrize("kind", [0, 1])
def test_gated_unit_at_the_ends_of_the_range(kind):
    big = [0.0, -0.0, 1e-30, -1e-30, 30.0, -30.0, 90.0, -90.0, 1e4, -1e4, 1e12, -1e12, 1e19, -1e19]
    g = torch.zeros(1, 32 * len(big), device="cuda")
    g[0, ::32] = torch.tensor(big, device="cuda")
    u = torch.ones_like(g)
    h, sg, su = torch.empty_like(g), store(1, g.shape[1], 8), store(1, g.shape[1], 8)
    B.abl_glu_forward(g, u, h, kind, 8, sg, su)
    want = R.act(f64(g), kind)[0]
    np.testing.assert_allclose(f64(h), np.nan_to_num(want), rtol=1e-5, atol=1e-9)
    dg, du = torch.empty_like(g), torch.empty_like(g)
    B.abl_glu_backward(u, sg, su, 8, dg, du, kind)
    assert torch.isfinite(dg).all() and torch.isfinite(du).all()
    pos = f64(g)[0, ::32]
    got = f64(dg)[0, ::32]
    np.testing.assert_allclose(got[pos >= 30], 1.0, rtol=1e-5)
    np.testing.assert_allclose(got[pos <= -30], 0.0, atol=1e-9)


def test_gated_unit_in_place():
    g, u = torch.randn(50, 70, device="cuda"), torch.randn(50, 70, device="cuda")
    h = torch.empty_like(g)
    B.abl_glu_forward(g, u, h, 0)
    g2 = g.clone()
    sg, su = store(50, 70, 8), store(50, 70, 8)
    B.abl_glu_forward(g2, u, g2, 0, 8, sg, su)
    assert torch.equal(g2, h)
    dg, du = torch.empty_like(g), torch.empty_like(g)
    B.abl_glu_backward(h, sg, su, 8, dg, du, 0)
    B.abl_glu_backward(g2, sg, su, 8, g2, u, 0)
    assert torch.equal(g2, dg) and torch.equal(u, du)


# ---- weight gradient ----------------------------------------------------------------------------------
WGRADS = [(0, 40, 24), (1, 1, 1), (1, 64, 64), (31, 33, 65), (32, 128, 128), (33, 100, 7), (100, 129, 130), (300, 257, 300), (1000, 64, 96),
          (5000, 40, 500), (2048, 256, 512), (1025, 520, 264)]


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype,flags", [(torch.float32, 0), (torch.float32, B.ABL_MATH_BF16), (torch.bfloat16, 0)])
@pytest.mark.parametrize("M,Cin,Cout", WGRADS)
def test_weight_gradient(M, Cin, Cout, dtype, flags, K):
    rng = np.random.default_rng(M + Cin + Cout)
    raw = R.pack(rng.standard_normal((M, Cin)), K) if M else np.zeros(128, np.uint8)
    x = R.unpack(raw, M, Cin, K)
    for pitch, scaled in ((0, False), (5, True), (8, True)):
        big = dev(rng.standard_normal((M, Cout + pitch)), dtype)
        dy = big[:, :Cout]
        scale = dev(rng.standard_normal(Cin) * 0.2 + 1, dtype) if scaled else None
        y = f64(dy.to(torch.bfloat16) if flags else dy)
        s = f64(scale)[:, None] if scaled else 1.0
        want = s * (x.T @ y)
        size = np.abs(s) * (np.abs(x).T @ np.abs(y))
        ws = torch.full((B.abl_ckpt_wgrad_scratch_bytes(M, Cin, Cout, dtype),), 0xFF, dtype=torch.uint8, device="cuda")
        dW = tensor(Cin, Cout)
        B.abl_ckpt_wgrad(torch.from_numpy(raw).cuda(), K, scale, dy, ws, dW, flags)
        hold(dW, want, size, U * (M + 8), torch.float32, "dW")
        acc = dW.clone()
        B.abl_ckpt_wgrad(torch.from_numpy(raw).cuda(), K, scale, dy, ws, acc, flags | B.ABL_ACCUM_DW)
        hold(acc, want + f64(dW), size + np.abs(f64(dW)), U * (M + 10), torch.float32, "dW accumulated")
        again = tensor(Cin, Cout)
        B.abl_ckpt_wgrad(torch.from_numpy(raw).cuda(), K, scale, dy, ws, again, flags)
        assert torch.equal(dW, again)


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradient_of_bf16_is_exact_in_its_operands(dtype):
    """Integers that every partial sum holds exactly: nothing is rounded anywhere."""
    rng = np.random.default_rng(11)
    M, Cin, Cout = 700, 200, 136
    x = rng.integers(-127, 128, (M, Cin)).astype(float)
    x[:, ::32] = 127                                   # every block has the scale 1
    x[:, 199] = 127
    y = rng.integers(-8, 9, (M, Cout)).astype(float)
    dW = tensor(Cin, Cout)
    ws = torch.empty(B.abl_ckpt_wgrad_scratch_bytes(M, Cin, Cout, dtype), dtype=torch.uint8, device="cuda")
    B.abl_ckpt_wgrad(torch.from_numpy(R.pack(x, 8)).cuda(), 8, None, dev(y, dtype), ws, dW)
    np.testing.assert_array_equal(f64(dW), x.T @ y)


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradient_shows_nan_and_infinities_where_they_belong(dtype):
    M, Cin, Cout = 70, 96, 80
    x = np.random.default_rng(12).standard_normal((M, Cin))
    x[10, 40] = np.nan
    dy = dev(np.random.default_rng(13).standard_normal((M, Cout)), dtype)
    dy[20, 7] = float("inf")
    dW = tensor(Cin, Cout)
    ws = torch.empty(B.abl_ckpt_wgrad_scratch_bytes(M, Cin, Cout, dtype), dtype=torch.uint8, device="cuda")
    B.abl_ckpt_wgrad(torch.from_numpy(R.pack(x, 8)).cuda(), 8, None, dy, ws, dW)
    bad = ~torch.isfinite(dW).cpu().numpy()
    want = np.zeros((Cin, Cout), bool)
    want[32:64] = True                                 # the block that holds the NaN
    want[:, 7] = True
    np.testing.assert_array_equal(bad, want)


def test_weight_gradient_of_a_slice_beyond_32_bits():
    M, Cin, Cout, pitch = 70, 64, 64, 1 << 26          # 70 rows 2^27 bytes apart
    big = torch.zeros(M * pitch, dtype=torch.bfloat16, device="cuda").view(M, pitch)
    rng = np.random.default_rng(14)
    y, x = rng.standard_normal((M, Cout)), rng.standard_normal((M, Cin))
    big[:, :Cout] = dev(y, torch.bfloat16)
    raw = R.pack(x, 8)
    dW = tensor(Cin, Cout)
    ws = torch.empty(B.abl_ckpt_wgrad_scratch_bytes(M, Cin, Cout, torch.bfloat16), dtype=torch.uint8, device="cuda")
    B.abl_ckpt_wgrad(torch.from_numpy(raw).cuda(), 8, None, big[:, :Cout], ws, dW)
    xq, yq = R.unpack(raw, M, Cin, 8), f64(big[:, :Cout])
    hold(dW, xq.T @ yq, np.abs(xq).T @ np.abs(yq), U * (M + 8), torch.float32, "dW")


# ---- how they are called ------------------------------------------------------------------------------
def test_calls_run_on_the_current_stream_and_in_a_graph():
    """All of them in turn, on a stream of their own and captured: every replay gives the eager result on new inputs."""
    M, C, F, K = 200, 320, 640, 8
    bf = dict(dtype=torch.bfloat16, device="cuda")
    r, b, gu, dh = (torch.empty(s, **bf) for s in ((M, C), (M, C), (M, 2 * F), (M, F)))
    w, gate = torch.ones(C, **bf), torch.full((2, C), 0.5, **bf)
    r2, n, h, dgu, dr, db = (torch.empty(s, **bf) for s in ((M, C), (M, C), (M, F), (M, 2 * F), (M, C), (M, C)))
    sb, sn, sg, su, sh = store(M, C, K), store(M, C, K), store(M, F, K), store(M, F, K), store(M, F, 8)
    rb, rn, dgate, dwp, dwq = tensor(M), tensor(M), tensor(2, C), tensor(C), tensor(C)
    dW, dW2 = tensor(C, 2 * F), tensor(F, C)
    ws = torch.empty(max(B.abl_resnorm_scratch_bytes(M, C), B.abl_ckpt_wgrad_scratch_bytes(M, C, 2 * F, torch.bfloat16),
                         B.abl_ckpt_wgrad_scratch_bytes(M, F, C, torch.bfloat16)), dtype=torch.uint8, device="cuda")
    outs = [r2, n, h, dgu, dr, db, sb, sn, sg, su, sh, rb, rn, dgate, dwp, dwq, dW, dW2]

    def work():
        B.abl_resnorm_forward(r, b, gate, 100, w, w, r2, n, K, sb, rb, sn, rn)
        B.abl_glu_forward(gu[:, :F], gu[:, F:], h, 0, K, sg, su)
        B.abl_glu_backward(dh, sg, su, K, dgu[:, :F], dgu[:, F:], 0, sh)
        B.abl_ckpt_wgrad(sh, 8, None, r2, ws, dW2)
        B.abl_ckpt_wgrad(sn, K, w, dgu, ws, dW)
        B.abl_resnorm_backward(n, r2, gate, 100, w, w, K, sb, rb, sn, rn, ws, dr, db, dgate, dwp, dwq)

    def fill(seed):
        torch.manual_seed(seed)
        for t in (r, b, gu, dh):
            t.copy_(torch.randn(t.shape, device="cuda"))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for seed in range(1, 5):
        fill(seed)
        work()
        torch.cuda.synchronize()
        eager = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(eager, outs):
            assert torch.equal(a, c)


def test_binding_refuses_wrong_tensors():
    x = torch.randn(4, 64, device="cuda")
    s = store(4, 64, 8)
    for bad in (lambda: B.abl_ckpt_pack(x.cpu(), 8, s), lambda: B.abl_ckpt_pack(x.t(), 8, s), lambda: B.abl_ckpt_pack(x, 8, s[:100]),
                lambda: B.abl_glu_forward(x, x.bfloat16(), x, 0), lambda: B.abl_glu_forward(x, x[:2], x, 0),
                lambda: B.abl_ckpt_wgrad(s, 8, x[0], x.bfloat16(), s, x),
                lambda: B.abl_resnorm_forward(x, x[:2], None, 0, None, x[0], x, x)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(B.AblError):
        B.abl_ckpt_pack(x.half(), 8, s)
    with pytest.raises(B.AblError):
        B.abl_ckpt_pack(x, 5, torch.zeros(10000, dtype=torch.uint8, device="cuda"))


# ---- what is not there, where a team has several rows --------------------------------------------------
SEVERAL = [(17000, 5), (17000, 40), (9000, 104), (4500, 1000), (3000, 1111), (2500, 1800), (2500, 2100), (2200, 4096), (1100, 4104), (1100, 8190), (1100, 8200),
           (9000, 4096)]   # M, C: every kind of team, whole and ragged rows, each team with two rows or more; the last beyond the caches


def same(a, b, what):
    assert a.keys() == b.keys(), what
    for k in a:
        assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), (what, k)


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C", SEVERAL)
def test_step_forward_without_a_branch_or_its_sum(M, C, dtype, K):
    """No b is a b of zeros, no r_out changes nothing else, and the rows of a team are as rows by themselves: bit for bit."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(C)
    r, b = (torch.randn(M, C, generator=gen, device="cuda").to(dtype) for _ in range(2))
    w, gate = ((torch.randn(n, C, generator=gen, device="cuda") * 0.3 + 1).to(dtype) for n in (1, 3))

    def call(r, b, gate, rows, post, k, want_r=True):
        m = len(r)
        keep = dict(n=torch.full_like(r, 7.0))
        if want_r:
            keep["r"] = torch.full_like(r, 7.0)
        if k:
            keep |= dict(sn=store(m, C, k), rn=tensor(m))
            if post or gate is not None:
                keep["sb"] = store(m, C, k)
            if post:
                keep["rb"] = tensor(m)
        B.abl_resnorm_forward(r, b, gate, rows, w[0] if post else None, w[0], keep.get("r"), keep["n"], k, keep.get("sb"), keep.get("rb"),
                              keep.get("sn"), keep.get("rn"), 0.75, 0.5)
        return keep

    for k in (0, K):
        none = call(r, None, None, 0, False, k)
        same(none, call(r, torch.zeros_like(b), None, 0, False, k), "no b")
        for with_b in (False, True):
            whole = call(r, b, gate, -(-M // 3), True, k) if with_b else none
            part = call(r, b, gate, -(-M // 3), True, k, want_r=False) if with_b else call(r, None, None, 0, False, k, want_r=False)
            same({n: v for n, v in whole.items() if n != "r"}, part, "no r_out")
        for first in (0, M - 120):   # (120 rows: a row a team)
            one = call(r[first: first + 120], None, None, 0, False, k)
            for n in ("n", "r") + (("rn",) if k else ()):
                assert torch.equal(none[n][first: first + 120], one[n]), n


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C", SEVERAL)
def test_step_backward_without_a_stream_a_branch_or_an_output(M, C, dtype, K):
    """No dr_out is one of zeros; without gate and norm db is dr where alpha is beta; without b, db or dr the others stay: bit for bit."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(C + 1)
    dn, dr_out, z, y = (torch.randn(M, C, generator=gen, device="cuda").to(dtype) for _ in range(4))
    rn, rb = (torch.exp(torch.randn(M, generator=gen, device="cuda") * 0.3) for _ in range(2))
    w, gate = ((torch.randn(n, C, generator=gen, device="cuda") * 0.3 + 1).to(dtype) for n in (1, 3))
    sn, sb = store(M, C, K), store(M, C, K)
    B.abl_ckpt_pack(z, K, sn)
    B.abl_ckpt_pack(y, K, sb)
    ws = torch.empty(B.abl_resnorm_scratch_bytes(M, C), dtype=torch.uint8, device="cuda")

    def call(dn, dr_out, full, has_b=True, drop=(), rows=slice(None), stores=None):
        m = len(dn)
        kn, kb = stores or (sn, sb)
        out = dict(dr=torch.full_like(dn, 7.0), db=torch.full_like(dn, 7.0), dw_pre=tensor(C))
        if full:
            out |= dict(dgate=tensor(3, C), dw_post=tensor(C))
        for k in drop if has_b else ("db",) + drop:
            del out[k]
        B.abl_resnorm_backward(dn, dr_out, gate if full else None, -(-m // 3) if full else 0, w[0] if full else None, w[0], K, kb if full else None,
                               rb[rows] if full else None, kn, rn[rows], ws, out.get("dr"), out.get("db"), out.get("dgate"), out.get("dw_post"),
                               out["dw_pre"], 0.5, 0.5, 0, has_b)
        return out

    without = lambda d, *names: {k: v for k, v in d.items() if k not in names}  # noqa: E731
    for full in (False, True):
        with_dr = call(dn, dr_out, full)
        same(call(dn, None, full), call(dn, torch.zeros_like(dn), full), "no dr_out")
        same(without(with_dr, "db"), call(dn, dr_out, full, drop=("db",)), "no db")
        same(without(with_dr, "dr"), call(dn, dr_out, full, drop=("dr",)), "no dr")
        if not full:
            assert torch.equal(with_dr["dr"], with_dr["db"])
            for d in (dr_out, None):
                same(without(call(dn, d, False), "db"), call(dn, d, False, has_b=False), "no b")
            same(without(call(dn, None, False), "db", "dr"), call(dn, None, False, has_b=False, drop=("dr",)), "no b, no dr")
    for first in (0, M - 60):   # rows by themselves
        part = slice(first, first + 60)
        one = store(60, C, K)
        B.abl_ckpt_pack(z[part], K, one)
        for d, e in ((dr_out, dr_out[part]), (None, None)):
            assert torch.equal(call(dn, d, False)["dr"][part], call(dn[part], e, False, rows=part, stores=(one, None))["dr"])


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Cin,Cout", [(64, 64), (130, 260), (100, 133), (300, 520)])
@pytest.mark.parametrize("M", [1, 31, 33, 65, 95, 161, 449])
def test_weight_gradient_takes_nothing_from_behind_its_rows(M, Cin, Cout, dtype, K):
    """Steps of 32 rows are asked for beyond the last: NaN lies there, behind dy and behind the store.  Small integers: the result is exact."""
    rng = np.random.default_rng(M + Cin)
    x = rng.integers(-4, 5, (M, Cin)).astype(float)
    x[:, ::32] = 4                                     # every block has a scale that its values are multiples of
    x[:, Cin - 1] = 4
    raw = R.pack(x, K)
    x = R.unpack(raw, M, Cin, K)
    y = rng.integers(-8, 9, (M, Cout)).astype(float)
    big = torch.full((M + 300, Cout), float("nan"), dtype=dtype, device="cuda")
    big[:M] = dev(y, dtype)
    behind = torch.full((raw.size + (1 << 16),), 0xFF, dtype=torch.uint8, device="cuda")
    behind[: raw.size] = torch.from_numpy(raw).cuda()
    ws = torch.full((B.abl_ckpt_wgrad_scratch_bytes(M, Cin, Cout, dtype),), 0xFF, dtype=torch.uint8, device="cuda")
    dW = tensor(Cin, Cout)
    B.abl_ckpt_wgrad(behind, K, None, big[:M], ws, dW)
    np.testing.assert_array_equal(f64(dW), x.T @ y)


@pytest.mark.parametrize("C", [40, 1111, 4096, 8200])
@pytest.mark.parametrize("center", [False, True])
def test_step_with_an_eps_below_the_least_normal_number(C, center):
    """Rows of zeros, of values whose squares vanish beside eps, and of values beside which eps vanishes.  (Ends: results to 2^-16 of them, as above;
    the subnormal eps itself is what its 32 bits hold.)"""
    eps = float(np.float32(1e-40))
    sign = np.where(np.arange(C) % 2 == 0, 1.0, -1.0)
    sign[-1] = 0.0 if C % 2 else sign[-1]              # (so that a row's sum is zero)
    x = np.stack([0 * sign, 2.0 ** -84 * sign, 2.0 ** -50 * sign, sign])
    r, w = dev(x, torch.float32), torch.ones(C, device="cuda")
    n, rn = tensor(4, C), tensor(4)
    B.abl_resnorm_forward(r, None, None, 0, None, w, None, n, 8, None, None, store(4, C, 8), rn, eps=eps, flags=B.ABL_NORM_CENTER if center else 0)
    want, rstd = R.norm(x, eps, center)
    np.testing.assert_allclose(f64(rn), rstd, rtol=2.0 ** -16)
    np.testing.assert_allclose(f64(n), want, rtol=2.0 ** -16, atol=0)


def test_binding_refuses_step_tensors_of_another_shape():
    """Enough elements are not enough: a transposed branch, a longer batch, a gate of other groups."""
    M, C, K, rows = 40, 64, 8, 10
    f = dict(device="cuda")
    good = dict(r=torch.randn(M, C, **f), b=torch.randn(M, C, **f), gate=torch.randn(4, C, **f), w=torch.ones(C, **f), r_out=tensor(M, C), n=tensor(M, C),
                dn=torch.randn(M, C, **f), dr_out=torch.randn(M, C, **f), dr=tensor(M, C), db=tensor(M, C), dgate=tensor(4, C))
    sb, sn, rb, rn, wp, wq = store(M, C, K), store(M, C, K), tensor(M), tensor(M), tensor(C), tensor(C)
    ws = torch.empty(B.abl_resnorm_scratch_bytes(M, C), dtype=torch.uint8, **f)

    def both(**kw):
        t = {**good, **kw}
        B.abl_resnorm_forward(t["r"], t["b"], t["gate"], rows, t["w"], t["w"], t["r_out"], t["n"], K, sb, rb, sn, rn)
        B.abl_resnorm_backward(t["dn"], t["dr_out"], t["gate"], rows, t["w"], t["w"], K, sb, rb, sn, rn, ws, t["dr"], t["db"], t["dgate"], wp, wq)

    both()
    for k, t in good.items():
        if k in ("gate", "dgate"):
            others = [t.new_zeros(5, C), t.new_zeros(3, C), t.new_zeros(2, 2 * C), t.flatten()]
        elif k == "w":
            others = [t.new_ones(C - 1), t.bfloat16()]
        elif k in ("r", "dn"):                                         # (they say how many rows there are: the others do not fit)
            others = [t.new_zeros(C, M), t.new_zeros(M + 1, C), t.new_zeros(2, M, C), t.flatten()]
        else:
            others = [t.new_zeros(C, M), t.new_zeros(M + 1, C), t.new_zeros(M, C + 1), t.flatten(), t.new_zeros(1, M, C)]
        for other in others:
            with pytest.raises(AssertionError):
                both(**{k: other})
    # no rows: the gate and its gradient have none that count
    none, keep = torch.empty(0, C, **f), store(1, C, K)
    B.abl_resnorm_forward(none, none, good["gate"], rows, good["w"], good["w"], none, none, K, keep, rb, keep, rn)
    B.abl_resnorm_backward(none, none, good["gate"], rows, good["w"], good["w"], K, keep, rb, keep, rn, ws, none, none, good["dgate"], wp, wq)
    assert bool((wp == 0).all()) and bool((wq == 0).all())


@pytest.mark.parametrize("far", [1 << 32, -(1 << 32), 1 << 40])
def test_binding_refuses_numbers_beyond_32_bits(far):
    """Not their low bits: K = 2^32 is not a call that keeps nothing, act = 2^32 is not the first unit, flags = 2^32 are not none."""
    M, C = 4, 64
    x, w, wp, wq, rn = torch.randn(M, C, device="cuda"), torch.ones(C, device="cuda"), tensor(C), tensor(C), tensor(M)
    s = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    for call in (lambda: B.abl_ckpt_pack(x, far + 8, s), lambda: B.abl_ckpt_unpack(s, far + 8, x), lambda: B.abl_glu_forward(x, x, x, far),
                 lambda: B.abl_glu_forward(x, x, x, 0, far), lambda: B.abl_glu_backward(x, s, s, 8, x, x, far),
                 lambda: B.abl_resnorm_forward(x, None, None, 0, None, w, x, x, flags=far), lambda: B.abl_resnorm_forward(x, None, None, 0, None, w, x, x, far),
                 lambda: B.abl_resnorm_backward(x, None, None, 0, None, w, 8, None, None, s, rn, s, x, x, None, None, wq, flags=far),
                 lambda: B.abl_ckpt_wgrad(s, 8, None, x, s, torch.empty(C, C, device="cuda"), far)):
        with pytest.raises(AssertionError):
            call()
