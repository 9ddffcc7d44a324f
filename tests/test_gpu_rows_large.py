"""Operators on rows of channels at the sizes where other kernels are chosen (large tiles, shares of the rows, passes that go by the
caches, rows of several pieces a thread), and the network that uses them together.  References in 64 bits with torch on the GPU from
the stores' values; tolerances as in test_gpu_rows.py: a sum of M products is off by at most M u of the sum of their magnitudes, u = 2^-24,
element-wise results by 2^-16 of their terms and half a unit of their type."""
import numpy as np
import pytest
import torch

from paper_1901_07988_amd import binding as B
from paper_1901_07988_amd import token_blocks as T
from tests import rows_reference as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def stored(x, K):
    """The store of x and its values in 64 bits."""
    s = torch.full((B.abl_ckpt_bytes(*x.shape, K),), 0xEE, dtype=torch.uint8, device="cuda")
    B.abl_ckpt_pack(x, K, s)
    v = torch.empty(x.shape, dtype=torch.float32, device="cuda")
    B.abl_ckpt_unpack(s, K, v)
    return s, v.double()


def within(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    assert not bool((off > 0).any()), (what, float((off / bound).max()))
    assert bool(torch.isfinite(got).all()), what


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype,flags", [(torch.bfloat16, 0), (torch.float32, 0), (torch.float32, B.ABL_MATH_BF16)])
@pytest.mark.parametrize("M,Cin,Cout", [
    (2048, 4096, 4096),     # large tiles, every unit with one
    (300, 4000, 4099),      # large tiles, ragged, few rows
    (8192, 1024, 1000),     # shares of the rows
    (8191, 2050, 1023),     # shares of large tiles, ragged
    (16384, 256, 264),      # many shares
    (16383, 250, 257),
    (33, 5000, 70),
])
def test_weight_gradient_of_large_products(M, Cin, Cout, dtype, flags, K):
    gen = generator(M + Cin)
    s, x = stored(normal(gen, M, Cin), K)
    dy = normal(gen, M, Cout, std=0.02, dtype=dtype)
    scale = normal(gen, Cin, std=0.2, dtype=dtype) + 1
    y = (dy.bfloat16() if flags else dy).double()
    w = scale.double()[:, None]
    want = w * torch.mm(x.t().contiguous(), y)
    size = w.abs() * torch.mm(x.abs().t().contiguous(), y.abs())
    ws = torch.full((B.abl_ckpt_wgrad_scratch_bytes(M, Cin, Cout, dtype),), 0xFF, dtype=torch.uint8, device="cuda")
    dW = torch.full((Cin, Cout), 7.0, device="cuda")
    B.abl_ckpt_wgrad(s, K, scale, dy, ws, dW, flags)
    within(dW, want, U * (M + 8) * size, "dW")
    again = torch.full((Cin, Cout), 7.0, device="cuda")
    B.abl_ckpt_wgrad(s, K, scale, dy, ws, again, flags)
    assert torch.equal(dW, again)
    B.abl_ckpt_wgrad(s, K, scale, dy, ws, again, flags | B.ABL_ACCUM_DW)
    within(again, want + dW.double(), U * (M + 10) * (size + dW.double().abs()), "dW accumulated")


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,Cin", [(4096, 4096), (500, 1001), (70, 70)])   # large tiles; shares, ragged; few rows
def test_weight_gradient_reads_every_code_and_scale(M, Cin, dtype, K):
    """dy is the identity: dW is the transposed store, exactly.  (Scales up to 2^115: no value overflows.)"""
    blocks = (Cin + 31) // 32
    gen = generator(K + M)
    s = torch.zeros(B.abl_ckpt_bytes(M, Cin, K), dtype=torch.uint8, device="cuda")
    codes = torch.randint(0, 256, (M * blocks, 4 * K), generator=gen, device="cuda").to(torch.uint8)
    if K == 8:
        codes[codes == 128] = 127   # (not a code)
    s[:codes.numel()] = codes.flatten()
    s[codes.numel():codes.numel() + M * blocks] = torch.randint(8, 243, (M * blocks,), generator=gen, device="cuda").to(torch.uint8)
    x = torch.empty((M, Cin), dtype=torch.float32, device="cuda")
    B.abl_ckpt_unpack(s, K, x)
    assert bool(torch.isfinite(x).all()) and int((x == 0).sum()) < x.numel() // 4
    dy = torch.eye(M, device="cuda").to(dtype)
    ws = torch.full((B.abl_ckpt_wgrad_scratch_bytes(M, Cin, M, dtype),), 0xFF, dtype=torch.uint8, device="cuda")
    dW = torch.full((Cin, M), 7.0, device="cuda")
    B.abl_ckpt_wgrad(s, K, None, dy, ws, dW)
    assert torch.equal(dW, x.t())


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weight_gradient_takes_a_slice_of_a_wide_tensor_and_leaves_nan_where_it_is(dtype, K):
    """Columns next to the slice hold NaN: a piece that reaches beyond the slice must not bring them into its sums."""
    gen = generator(3)
    M, Cin, Cout, first, wide = 515, 300, 203, 5, 230
    x = normal(gen, M, Cin)
    x[7, 100] = float("nan")
    s = torch.zeros(B.abl_ckpt_bytes(M, Cin, K), dtype=torch.uint8, device="cuda")
    B.abl_ckpt_pack(x, K, s)
    v = torch.empty(M, Cin, device="cuda")
    B.abl_ckpt_unpack(s, K, v)
    big = torch.full((M, wide), float("nan"), dtype=dtype, device="cuda")
    dy = big[:, first: first + Cout]
    dy.copy_(normal(gen, M, Cout, dtype=dtype))
    ws = torch.empty(B.abl_ckpt_wgrad_scratch_bytes(M, Cin, Cout, dtype), dtype=torch.uint8, device="cuda")
    dW = torch.full((Cin, Cout), 7.0, device="cuda")
    B.abl_ckpt_wgrad(s, K, None, dy, ws, dW)
    bad = torch.isnan(dW).cpu().numpy()
    want = np.zeros((Cin, Cout), bool)
    want[96:128] = True                                  # the block with the NaN
    np.testing.assert_array_equal(bad, want)
    ok = torch.ones(Cin, dtype=torch.bool, device="cuda")
    ok[96:128] = False
    a, y = v[:, ok].double(), dy.double()
    within(dW[ok], torch.mm(a.t().contiguous(), y), U * (M + 8) * torch.mm(a.abs().t().contiguous(), y.abs()), "dW")


@pytest.mark.parametrize("M,Cin,Cout,pitch,dtype,K", [
    (40000, 96, 64, 1 << 16, torch.bfloat16, 8),         # shares of the rows are near enough
    (5000, 4096, 4096, 1 << 19, torch.bfloat16, 8),      # products of 1280 rows, one after the other
    (5000, 4000, 4099, 1 << 19, torch.float32, 4),       # of 640 rows, ragged
    (20001, 2050, 2007, 1 << 18, torch.bfloat16, 4),     # with shares of their own
    (5000, 1 << 19, 16, 16, torch.bfloat16, 4),          # a wide input
    (300, 70, 40, 1 << 23, torch.bfloat16, 8),           # farther apart than products reach
])
def test_weight_gradient_of_rows_whose_offsets_pass_31_bits(M, Cin, Cout, pitch, dtype, K):
    gen = generator(M + Cin)
    s, x = stored(normal(gen, M, Cin), K)
    big = torch.full((M, pitch), float("nan"), dtype=dtype, device="cuda")
    dy = big[:, :Cout]
    dy.copy_(normal(gen, M, Cout, std=0.02))
    scale = normal(gen, Cin, std=0.2, dtype=dtype) + 1
    w, y = scale.double()[:, None], dy.double()
    want = w * torch.mm(x.t().contiguous(), y)
    size = w.abs() * torch.mm(x.abs().t().contiguous(), y.abs())
    ws = torch.full((B.abl_ckpt_wgrad_scratch_bytes(M, Cin, Cout, dtype),), 0xFF, dtype=torch.uint8, device="cuda")
    assert ws.numel() <= 256 << 20
    dW = torch.full((Cin, Cout), 7.0, device="cuda")
    B.abl_ckpt_wgrad(s, K, scale, dy, ws, dW)
    within(dW, want, U * (M + 8) * size, "dW")
    again = dW.clone()
    B.abl_ckpt_wgrad(s, K, scale, dy, ws, again, B.ABL_ACCUM_DW)
    within(again, want + dW.double(), U * (M + 10) * (size + dW.double().abs()), "dW accumulated")


@pytest.mark.parametrize("M,C", [(70, 200), (600, 1111)])
def test_one_gate_row_for_any_number_of_rows(M, C):
    """gate_rows far beyond the rows: as one group of them all."""
    gen, K = generator(C), 8
    r, b, dn, dr_out = (normal(gen, M, C) for _ in range(4))
    gate, w = normal(gen, 1, C), normal(gen, C)
    results = []
    for rows in (M, 2 ** 62, 2 ** 63 - 1):
        sb, sn = (torch.zeros(B.abl_ckpt_bytes(M, C, K), dtype=torch.uint8, device="cuda") for _ in range(2))
        rb, rn = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        r2, n, dr, db = (torch.empty_like(r) for _ in range(4))
        dg, dp, dq = torch.empty(1, C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        ws = torch.empty(B.abl_resnorm_scratch_bytes(M, C), dtype=torch.uint8, device="cuda")
        B.abl_resnorm_forward(r, b, gate, rows, w, w, r2, n, K, sb, rb, sn, rn)
        B.abl_resnorm_backward(dn, dr_out, gate, rows, w, w, K, sb, rb, sn, rn, ws, dr, db, dg, dp, dq)
        results.append((r2, n, sb, sn, rb, rn, dr, db, dg, dp, dq))
    for other in results[1:]:
        for a, c in zip(results[0], other):
            assert torch.equal(a, c)


@pytest.mark.parametrize("M,C,K,gate_rows", [(8192, 4096, 8, 2048), (4096, 8192, 4, 1), (70000, 1500, 8, 0), (9000, 4104, 8, 9000)])
def test_step_on_tensors_beyond_the_caches(M, C, K, gate_rows):
    gen = generator(C)
    bf = torch.bfloat16
    r, b = normal(gen, M, C, dtype=bf), normal(gen, M, C, dtype=bf)
    gate = normal(gen, -(-M // gate_rows), C, std=0.3, dtype=bf) if gate_rows else None
    w_post, w_pre = normal(gen, C, std=0.2, dtype=bf) + 1, normal(gen, C, std=0.2, dtype=bf) + 1
    r_out, n = torch.empty_like(r), torch.empty_like(r)
    sb, sn = (torch.empty(B.abl_ckpt_bytes(M, C, K), dtype=torch.uint8, device="cuda") for _ in range(2))
    rb, rn = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    B.abl_resnorm_forward(r, b, gate, gate_rows, w_post, w_pre, r_out, n, K, sb, rb, sn, rn)
    y, z = torch.empty(M, C, device="cuda"), torch.empty(M, C, device="cuda")
    B.abl_ckpt_unpack(sb, K, y)
    B.abl_ckpt_unpack(sn, K, z)
    at = torch.cat([torch.arange(0, M, max(1, M // 50), device="cuda"), torch.tensor([M - 1], device="cuda")])
    f = {k: t[at].double().cpu().numpy() for k, t in dict(r=r, b=b, r_out=r_out, n=n, y=y, z=z, rb=rb, rn=rn).items()}
    g = None if gate is None else gate.double().cpu().numpy()[at.cpu().numpy() // gate_rows]
    wp, wq = w_post.double().cpu().numpy(), w_pre.double().cpu().numpy()
    want = R.step_forward(f["r"], f["b"], g, 1, wp, wq, 1.0, 1.0, 1e-5, False)
    for k, ref in (("r_out", want["r"]), ("n", want["n"])):
        assert (np.abs(f[k] - ref) <= 2.0 ** -8 * 1.01 * np.abs(ref) + 2.0 ** -14).all(), k
    for k, ref in (("rb", want["rstd_b"]), ("rn", want["rstd_n"])):
        np.testing.assert_allclose(f[k], ref, rtol=2.0 ** -16)
    for k, ref in (("y", want["y"]), ("z", want["z"])):   # the next code at most: a quarter of the value in 4 bits, the step of the block in 8
        step = np.repeat(np.abs(R.blocked(ref)).max(-1), 32, axis=1)[:, :C] / (63 if K == 8 else 3)
        assert (np.abs(f[k] - ref) <= step).all(), k
        assert (R.unpack(R.pack(ref, K), len(at), C, K) != f[k]).mean() < 1e-3, k
    # backward, from the stores' values
    dn, dr_out = normal(gen, M, C, std=0.02, dtype=bf), normal(gen, M, C, std=0.02, dtype=bf)
    dr, db = torch.empty_like(r), torch.empty_like(r)
    dgate = torch.empty(gate.shape, device="cuda") if gate_rows else None
    dwp, dwq = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = torch.full((B.abl_resnorm_scratch_bytes(M, C),), 0xFF, dtype=torch.uint8, device="cuda")
    B.abl_resnorm_backward(dn, dr_out, gate, gate_rows, w_post, w_pre, K, sb, rb, sn, rn, ws, dr, db, dgate, dwp, dwq)
    h = {k: t[at].double().cpu().numpy() for k, t in dict(dn=dn, dr_out=dr_out, dr=dr, db=db).items()}
    ref = R.step_backward(h["dn"], h["dr_out"], f["y"], f["rb"], f["z"], f["rn"], g, 1, wp, wq, 1.0, 1.0, False)
    for k in ("dr", "db"):
        terms = 2.0 ** -16 * (np.abs(ref[k]) + np.abs(ref[k]).max(1, keepdims=True))
        assert (np.abs(h[k] - ref[k]) <= 2.0 ** -8 * 1.01 * np.abs(ref[k]) + 4 * terms).all(), k
    # sums over all rows, in parts of them
    sums = [torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(4)]
    gsum = torch.zeros(gate.shape, dtype=torch.float64, device="cuda") if gate_rows else None
    for i in range(0, M, 2048):
        p = slice(i, min(i + 2048, M))
        d, zz, yy = dn[p].double(), z[p].double(), y[p].double()
        v = d * w_pre.double()
        D = dr_out[p].double() + rn[p].double()[:, None] * (v - zz * (v * zz).mean(1, keepdim=True))
        sums[0] += (d * zz).sum(0)
        sums[1] += (d * zz).abs().sum(0)
        group = torch.arange(p.start, p.stop, device="cuda") // gate_rows if gate_rows else None
        e = D * gate.double()[group] if gate_rows else D
        sums[2] += (e * yy).sum(0)
        sums[3] += (e * yy).abs().sum(0)
        if gate_rows:
            gsum.index_add_(0, group, D * yy * w_post.double())
    terms = 2.0 ** -16 + U * M
    within(dwq, sums[0], terms * sums[1], "dw_pre")
    within(dwp, sums[2], terms * sums[3], "dw_post")
    if gate_rows:
        size = sums[3].max() if gate_rows > 1 else gsum.abs().max()
        within(dgate, gsum, terms * size.expand_as(gsum), "dgate")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_step_of_the_widest_rows_that_are_not_whole_pieces(dtype):
    M, C, K = 5, 16381, 8
    gen = generator(1)
    r, b = normal(gen, M, C, dtype=dtype), normal(gen, M, C, dtype=dtype)
    w = normal(gen, C, std=0.2, dtype=dtype) + 1
    guard = torch.full((M + 2, C), 7.0, dtype=dtype, device="cuda")
    n = guard[1: M + 1]
    sb, sn = (torch.empty(B.abl_ckpt_bytes(M, C, K), dtype=torch.uint8, device="cuda") for _ in range(2))
    rb, rn = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    B.abl_resnorm_forward(r, b, None, 0, w, w, None, n, K, sb, rb, sn, rn)
    want = R.step_forward(*(t.double().cpu().numpy() for t in (r, b)), None, 0, *(w.double().cpu().numpy(),) * 2, 1.0, 1.0, 1e-5, False)
    got = n.double().cpu().numpy()
    half = 2.0 ** -8 * 1.01 if dtype == torch.bfloat16 else 0.0
    assert (np.abs(got - want["n"]) <= half * np.abs(want["n"]) + 2.0 ** -14).all()
    assert bool((guard[0] == 7).all()) and bool((guard[M + 1] == 7).all())
    dn = normal(gen, M, C, std=0.02, dtype=dtype)
    dr = torch.full((M + 2, C), 7.0, dtype=dtype, device="cuda")
    dwp, dwq = torch.full((C + 8,), 7.0, device="cuda"), torch.full((C + 8,), 7.0, device="cuda")
    db = torch.empty_like(r)
    ws = torch.empty(B.abl_resnorm_scratch_bytes(M, C), dtype=torch.uint8, device="cuda")
    B.abl_resnorm_backward(dn, None, None, 0, w, w, K, sb, rb, sn, rn, ws, dr[1: M + 1], db, None, dwp[:C], dwq[:C])
    y, z = (R.unpack(t.cpu().numpy(), M, C, K) for t in (sb, sn))
    ref = R.step_backward(dn.double().cpu().numpy(), None, y, rb.double().cpu().numpy(), z, rn.double().cpu().numpy(), None, 0,
                          *(w.double().cpu().numpy(),) * 2, 1.0, 1.0, False)
    for k, t in (("dr", dr[1: M + 1]), ("db", db)):
        terms = 2.0 ** -14 * np.abs(ref[k]).max(1, keepdims=True)
        assert (np.abs(t.double().cpu().numpy() - ref[k]) <= half * np.abs(ref[k]) + terms).all(), k
    for t, k in ((dwp, "dw_post"), (dwq, "dw_pre")):
        assert (np.abs(t[:C].double().cpu().numpy() - ref[k]) <= 2.0 ** -14 * np.abs(ref[k]).max()).all(), k
        assert bool((t[C:] == 7).all())
    assert bool((dr[0] == 7).all()) and bool((dr[M + 1] == 7).all())


# ---- the network --------------------------------------------------------------------------------------
def test_network_gradients_are_those_of_the_exact_one_up_to_the_stores():
    """What a store leaves out: 8 bits 0.7 %, 4 bits 10 % of a block's standard deviation, and bf16 0.2 % at each of some twenty tensors on a
    path of two blocks; relative errors of gradients are held to three times the root of the sum of squares."""
    tokens, C, F, layers = 1000, 256, 352, 2
    fresh = lambda: T.random_parameters(layers, C, F, 3, seed=5)  # noqa: E731
    for act in (B.ABL_ACT_SILU, B.ABL_ACT_GELU):
        exact = T.ExactNet(*fresh(), tokens, act=act, alpha=0.9, beta=0.8)
        x, dn = T.batch(tokens, C, 1), T.batch(tokens, C, 2)
        out = exact.forward(x)
        exact.backward(dn)
        for K, bound in ((8, 3 * (8 * 0.007 ** 2 + 20 * 0.002 ** 2) ** 0.5), (4, 3 * (8 * 0.1 ** 2) ** 0.5)):
            net = T.TokenNet(*fresh(), tokens, K, act=act, alpha=0.9, beta=0.8)
            got = net.forward(x)
            assert T.relative(got, out.detach()) < 3 * (20 * 0.002 ** 2) ** 0.5      # the forward pass does not depend on K
            net.backward(dn)
            for name, e in T.gradient_errors(net, exact).items():
                assert e < bound, (K, act, name, e)
            assert T.relative(net.g_last, exact.g_last) < bound
            first = [{k: v.clone() for k, v in g.items()} for g in net.grads]
            net.backward(dn, accumulate=True)
            for a, b in zip(net.grads, first):
                for k in ("W1", "W2"):
                    assert torch.equal(a[k], 2 * b[k]), k                            # twice the same sum
                assert torch.equal(a["gate"], b["gate"])


def test_network_trains_as_the_exact_one():
    curves = T.main(["--layers", "2", "--tokens", "512", "--channels", "128", "--width", "192", "--steps", "25", "--samples", "2"])
    exact = np.array(curves["exact"])
    assert exact[-1] < 0.95 * exact[0]
    np.testing.assert_allclose(curves["K=8"], exact, rtol=0.01)
    np.testing.assert_allclose(curves["K=4"], exact, rtol=0.06)


def empty_store(M, C, K):
    return torch.empty(B.abl_ckpt_bytes(M, C, K), dtype=torch.uint8, device="cuda")


def test_step_on_tensors_of_more_than_4_gb():
    """The last rows, as a tensor of their own, give the same bits."""
    M, C, K, tail = 300001, 8192, 8, 65
    gen = generator(5)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    r, b, dn, dr_out = (torch.randn(M, C, generator=gen, **bf) for _ in range(4))
    gate, w = normal(gen, 1, C, dtype=torch.bfloat16), normal(gen, C, dtype=torch.bfloat16)

    def step(r, b, dn, dr_out):
        M = len(r)
        sb, sn, rb, rn = empty_store(M, C, K), empty_store(M, C, K), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        r2, n, dr, db = (torch.empty_like(r) for _ in range(4))
        dg, dp, dq = torch.empty(1, C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        ws = torch.empty(B.abl_resnorm_scratch_bytes(M, C), dtype=torch.uint8, device="cuda")
        B.abl_resnorm_forward(r, b, gate, M, w, w, r2, n, K, sb, rb, sn, rn)
        B.abl_resnorm_backward(dn, dr_out, gate, M, w, w, K, sb, rb, sn, rn, ws, dr, db, dg, dp, dq)
        values = torch.empty_like(r)
        B.abl_ckpt_unpack(sn, K, values)
        return r2, n, rb, rn, dr, db, values

    whole = [t[-tail:].clone() for t in step(r, b, dn, dr_out)]
    part = step(*(t[-tail:].clone() for t in (r, b, dn, dr_out)))
    for a, c in zip(whole, part):
        assert torch.equal(a, c)


def test_gated_unit_on_tensors_of_more_than_4_gb():
    M, F, K, tail = 70001, 32768, 8, 33
    gen = generator(6)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    gu, dh = torch.randn(M, 2 * F, generator=gen, **bf), torch.randn(M, F, generator=gen, **bf)

    def unit(gu, dh):
        M = len(gu)
        sg, su, sh = (empty_store(M, F, K) for _ in range(3))
        h, dgu, values = torch.empty_like(dh), torch.empty_like(gu), torch.empty_like(dh)
        B.abl_glu_forward(gu[:, :F], gu[:, F:], h, B.ABL_ACT_SILU, K, sg, su)
        B.abl_glu_backward(dh, sg, su, K, dgu[:, :F], dgu[:, F:], B.ABL_ACT_SILU, sh)
        B.abl_ckpt_unpack(sh, K, values)
        return h, dgu, values

    whole = [t[-tail:].clone() for t in unit(gu, dh)]
    for a, c in zip(whole, unit(gu[-tail:].clone(), dh[-tail:].clone())):
        assert torch.equal(a, c)


@pytest.mark.parametrize("M,C,K,gate_rows", [
    (3000, 1025, 8, 3000), (2500, 1280, 8, 500), (2000, 1529, 4, 1), (3000, 1536, 8, 0), (1500, 1537, 8, 300),   # teams of 192 threads, and of 256 beside them
    (40000, 1280, 8, 2000),                                                                                      # beyond the caches
    (1000, 500, 8, 250), (1000, 513, 8, 1), (1000, 1016, 4, 0),
])
def test_step_at_the_widths_where_teams_change(M, C, K, gate_rows):
    test_step_on_tensors_beyond_the_caches(M, C, K, gate_rows)


@pytest.mark.parametrize("tokens,samples", [(10, 6), (9, 4), (130, 64), (3, 5)])
def test_network_of_more_gate_rows_than_runs_of_tokens(tokens, samples):
    """Rows of the gates that no token takes: their gradients are zero, whatever lay in the memory, and an update leaves them as they are."""
    C, F = 64, 96
    used = -(-tokens // -(-tokens // samples))
    assert used < samples
    dirt = [torch.full((samples, C), float("nan"), device="cuda") for _ in range(64)]    # (what freed memory may hold)
    del dirt
    net = T.TokenNet(*T.random_parameters(2, C, F, samples, seed=3), tokens, 8)
    exact = T.ExactNet(*T.random_parameters(2, C, F, samples, seed=3), tokens)
    x, dn = T.batch(tokens, C, 1), T.batch(tokens, C, 2)
    for n in (net, exact):
        n.forward(x)
        n.backward(dn)
    before = [p["gate"].clone() for p in net.master]
    for g, e in zip(net.grads, exact.grads):
        assert bool((g["gate"][used:] == 0).all()) and bool((e["gate"][used:] == 0).all())
        assert bool((g["gate"][:used] != 0).any(1).all())
    net.update(0.1)
    for p, b in zip(net.master, before):
        assert torch.equal(p["gate"][used:], b[used:]) and not torch.equal(p["gate"][:used], b[:used])


@pytest.mark.parametrize("parts", [2, 3])
def test_network_updates_with_the_sum_of_a_batch_in_parts(parts):
    """Against the parts' own gradients, added here: sums of two or three numbers in fp32, and W1 and W2 in the kernel's order."""
    tokens, C, F, K, lr = 70, 64, 96, 8, 0.5
    fresh = lambda: T.TokenNet(*T.random_parameters(2, C, F, 3, seed=4), tokens, K)  # noqa: E731
    net, sums, size = fresh(), None, None
    before = [{k: v.clone() for k, v in p.items()} for p in net.master]
    for i in range(parts):
        x, dn = T.batch(tokens, C, 10 + i), T.batch(tokens, C, 20 + i)
        alone = fresh()
        for n in (net, alone):
            n.forward(x)
        net.backward(dn, accumulate=i > 0)
        alone.backward(dn)
        g = [{k: v.double() for k, v in d.items()} for d in alone.grads]
        sums = g if sums is None else [{k: a[k] + b[k] for k in a} for a, b in zip(sums, g)]
        size = [{k: v.abs() for k, v in d.items()} for d in g] if size is None else [{k: a[k] + b[k].abs() for k in a} for a, b in zip(size, g)]
    net.update(lr)
    for p, b, s, m in zip(net.master, before, sums, size):
        for k in T.PARAMETERS:
            within(p[k], b[k].double() - lr * s[k], (2 * parts + 4) * U * (b[k].abs() + lr * m[k]), k)
    net.backward(dn)                                   # a new batch takes nothing of the old one
    assert not net.earlier


@pytest.mark.parametrize("parts", [1, 2])
def test_network_updates_the_last_norms_weight(parts):
    tokens, C, F, lr = 70, 64, 96, 0.5
    fresh = lambda: T.random_parameters(2, C, F, 3, seed=4)  # noqa: E731
    net, exact = T.TokenNet(*fresh(), tokens, 8), T.ExactNet(*fresh(), tokens)
    before, total = net.w_last32.clone(), 0.0
    for i in range(parts):
        net.forward(T.batch(tokens, C, 10 + i))
        net.backward(T.batch(tokens, C, 20 + i), accumulate=i > 0)
        total = total + net.g_last.double()
    net.update(lr)
    within(net.w_last32, before.double() - lr * total, 8 * U * (before.abs() + lr * total.abs() + 1), "w_last")
    assert torch.equal(net.w_last, net.w_last32.bfloat16())
    exact.forward(T.batch(tokens, C, 10))
    exact.backward(T.batch(tokens, C, 20))
    exact.update(lr)
    within(exact.w_last32, before.double() - lr * exact.g_last.double(), 8 * U * (before.abs() + lr * exact.g_last.abs()), "w_last, exact")


@pytest.mark.parametrize("K", [4, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,C,gate_rows", [
    (17000, 5, 0), (17000, 5, 700), (17001, 40, 3), (17001, 40, 1), (5000, 104, 5000), (9001, 500, 450), (4500, 1000, 2), (3000, 1111, 1), (3001, 1111, 1300),
    (40000, 1280, 2000), (70000, 1500, 0), (2500, 1800, 2500), (2500, 2100, 7), (8192, 4096, 2048), (8191, 4096, 33), (8191, 4096, 31), (9000, 4104, 9000),
    (4096, 8192, 1), (1100, 8190, 500), (1100, 8200, 0), (1101, 8200, 2), (700, 16381, 100)])
def test_sums_over_the_rows_of_a_step_are_exact_for_whole_numbers(M, C, gate_rows, dtype, K):
    """Stores of whole numbers, gradients of whole numbers, weights and gates of powers of two: no sum is rounded, in whatever order, so that a row or
    a share that is missing, doubled or in another group is seen.  dw_pre with no dr_out; dw_post and dgate with no dn, where D is dr_out."""
    gen = generator(M + C)
    top = 127 if K == 8 else 6

    def whole(lo, hi, *shape):
        return torch.randint(lo, hi + 1, shape, generator=gen, device="cuda").float()

    def kept():
        x = whole(-4, 4, M, C)
        x[:, ::32] = top                     # (the scale of every block is 1)
        s, v = stored(x, K)
        assert torch.equal(v.float(), x)
        return s, v

    (sn, z), (sb, y) = kept(), kept()
    one = torch.ones(M, device="cuda")
    G = -(-M // gate_rows) if gate_rows else 0
    w_post, w_pre = (torch.exp2(whole(-1, 1, C)).to(dtype) for _ in range(2))
    gate = torch.exp2(whole(-1, 1, G, C)).to(dtype) if G else None
    ws = torch.full((B.abl_resnorm_scratch_bytes(M, C),), 0xFF, dtype=torch.uint8, device="cuda")
    group = torch.arange(M, device="cuda") // gate_rows if G else None
    for dn, dr_out in ((whole(-2, 2, M, C), None), (torch.zeros(M, C, device="cuda"), whole(-2, 2, M, C))):
        dwp, dwq = torch.full((C,), 7.0, device="cuda"), torch.full((C,), 7.0, device="cuda")
        dgate = torch.full((G, C), 7.0, device="cuda") if G else None
        dr, db = torch.empty(M, C, dtype=dtype, device="cuda"), torch.empty(M, C, dtype=dtype, device="cuda")
        B.abl_resnorm_backward(dn.to(dtype), None if dr_out is None else dr_out.to(dtype), gate, gate_rows, w_post, w_pre, K, sb, one, sn, one, ws, dr, db,
                               dgate, dwp, dwq, 1.0, 0.5)
        assert torch.equal(dwq.double(), (dn.double() * z).sum(0)), "dw_pre"
        if dr_out is None:
            continue
        assert torch.equal(dr.float(), dr_out)
        e = 0.5 * dr_out.double() * y
        assert torch.equal(dwp.double(), (e * gate.double()[group] if G else e).sum(0)), "dw_post"
        if G:
            want = torch.zeros(G, C, dtype=torch.float64, device="cuda").index_add_(0, group, e * w_post.double())
            assert torch.equal(dgate.double(), want), "dgate"
