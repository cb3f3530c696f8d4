"""The residual block's operators against plain 64-bit implementations: norm, 8-bit forms, 8-bit product, weight gradient.

Tolerances come from the operations, with u = 2^-24 (fp32 rounding) and 2^-9 (bf16 rounding, half an ulp):
  - a sum of squares or products over a row passes at most 64 additions in a lane, 5 shuffles and 32 warps: 128 u of the sum
    of magnitudes covers it and the few operations after it;
  - a bf16 output adds 2^-9 of its value, taken as 2^-8 (the value may have been moved across a rounding boundary);
  - an e4m3 value is within 2^-4 of what it stands for, or within half its smallest step (2^-10 scales);
  - the tensor cores add 32 products an instruction: K/32 + K/128 additions, each rounding (or truncating) to no worse than
    2^-22 of the sum of magnitudes so far."""
import numpy as np
import pytest
import torch

from paper_2406_17611_b200 import binding as vb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn


def ld_of(F, dtype, extra=0):
    v = 16 // torch.empty((), dtype=dtype).element_size()
    return ((F + v - 1) // v + extra) * v


def matrix(x, dtype, extra=0, fill=float("nan")):
    """[rows x ld] device matrix with x in its first columns and `fill` in the padding, which nothing may read as data."""
    m = torch.full((x.shape[0], ld_of(x.shape[1], dtype, extra)), fill, device=DEV).to(dtype)
    m[:, :x.shape[1]] = x.to(dtype)
    return m


def d64(t, F=None):
    return t[:, :F].to(torch.float64)


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(rows, F, g, scale=1.0):
    return torch.randn((rows, F), generator=g, device=DEV) * scale


def roundoff(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2 * U


def spread(s, F):
    return s.t().to(torch.float64).repeat_interleave(128, dim=1)[:, :F]


def check_eight(q, s, y, err):
    """q, s: 8-bit form; y: what it stands for in 64 bits, known to within err (elementwise)."""
    F = y.shape[1]
    nb = (F + 127) // 128
    pad = torch.nn.functional.pad(y.abs() + err, (0, nb * 128 - F)).view(y.shape[0], nb, 128).amax(2)
    low = torch.nn.functional.pad((y.abs() - err).clamp_min(0), (0, nb * 128 - F)).view(y.shape[0], nb, 128).amax(2)
    s64 = s.t().to(torch.float64)
    assert bool((s64 <= (pad / 448).clamp_min(2.0 ** -126) * (1 + 4 * U)).all())
    assert bool((s64 >= (low / 448).clamp_min(2.0 ** -126) * (1 - 4 * U)).all())
    sc = spread(s, F)
    v = d64(q, F) * sc
    assert bool(torch.isfinite(v).all())
    bound = torch.maximum((y.abs() + err) * 2.0 ** -4, sc * 2.0 ** -10) * (1 + 1e-5) + err
    assert bool(((v - y).abs() <= bound).all()), float(((v - y).abs() - bound).max())


# ------------------------------------------------------------------------------------------ norm
NORM_SHAPES = [(1, 1), (1, 256), (3, 7), (33, 8), (5, 47), (300, 64), (257, 100), (1000, 128), (129, 129), (64, 256), (700, 256),
               (41, 511), (100, 602), (9, 1000), (17, 1024), (6, 2047), (5, 4096), (3, 8192), (2, 16384)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,F", NORM_SHAPES)
def test_norm_forward(rows, F, dtype):
    g = gen(rows * 31 + F)
    for residual, gain, quantize in ((True, True, True), (False, False, False), (True, False, True), (False, True, True)):
        x, r = randn(rows, F, g, 3.0), randn(rows, F, g)
        x[:, ::5] *= 20
        if rows > 2:
            x[1], r[1] = 0, 0                       # a row of zeros: an isolated node after a ReLU
        X, R = matrix(x, dtype, 1), matrix(r, dtype) if residual else None
        G = 1 + 0.3 * torch.randn(F, generator=g, device=DEV) if gain else None
        out = vb.varco_norm_fwd(X, F, gain=G, residual=R, eps=1e-6, quantize=quantize)
        h = d64(X, F) + (d64(R, F) if residual else 0)
        rstd = 1 / ((h * h).mean(1) + 1e-6).sqrt()
        y = h * rstd[:, None] * (G.double() if gain else 1)
        assert bool(((out.rstd.double() - rstd).abs() <= 128 * U * rstd).all())
        if residual:
            assert bool(((d64(out.H, F) - h).abs() <= (U + roundoff(dtype)) * h.abs()).all())
            assert not out.H[:, F:].any()
        else:
            assert out.H is None
        # a sum h that cancels is off by u of its addends, and that is carried through the gain
        err = 128 * U * (y.abs() + (d64(X, F).abs() + (d64(R, F).abs() if residual else 0)) * rstd[:, None] * (G.abs().double() if gain else 1) / 64)
        assert bool(((d64(out.Y, F) - y).abs() <= err + roundoff(dtype) * y.abs()).all())
        assert not out.Y[:, F:].any()
        if quantize:
            check_eight(out.Y8, out.scales, y, err)
        else:
            assert out.Y8 is None and out.scales is None


def test_norm_forward_only_eight_bits_and_repeatable():
    g = gen(3)
    X, G = matrix(randn(500, 200, g), torch.bfloat16), torch.ones(200, device=DEV)
    a = vb.varco_norm_fwd(X, 200, gain=G, quantize=True)
    b = vb.varco_norm_fwd(X, 200, gain=G, quantize=True, keep=False)
    assert b.Y is None and torch.equal(a.Y8.view(torch.uint8)[:, :200], b.Y8.view(torch.uint8)[:, :200]) and torch.equal(a.scales, b.scales)


def test_norm_not_finite_rows_stay_in_their_rows():
    g = gen(4)
    x = randn(6, 300, g)
    x[1, 3], x[3, 299], x[4, 0] = float("nan"), float("inf"), -float("inf")
    out = vb.varco_norm_fwd(matrix(x, torch.float32), 300, quantize=True)
    bad = [1, 3, 4]
    good = [0, 2, 5]
    assert bool(torch.isfinite(out.Y[good]).all()) and bool(torch.isfinite(out.scales[:, good]).all())
    assert bool(torch.isnan(out.Y[1, :300]).all()) and bool(torch.isnan(out.Y[3, 299])) and bool(torch.isnan(out.Y[4, 0]))
    v = d64(out.Y8, 300) * spread(out.scales, 300)
    assert bool(torch.isfinite(v[good]).all())
    assert bool(torch.isnan(v[1]).all()) and bool(torch.isnan(v[3, 299])) and bool(torch.isnan(v[4, 0]))
    assert not out.Y[bad][:, 300:].any()


def test_norm_empty():
    X = torch.zeros((0, 64), device=DEV)
    out = vb.varco_norm_fwd(X, 64, residual=X, quantize=True)
    assert out.Y.shape == (0, 64) and out.scales.shape == (1, 0)
    ws = vb.varco_ops_workspace(64)
    r = vb.varco_norm_bwd(X, X, torch.zeros(0, device=DEV), 64, gain=torch.ones(64, device=DEV), workspace=ws)
    assert not r.dgain.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,F", NORM_SHAPES + [(40000, 40)])
def test_norm_backward(rows, F, dtype):
    g = gen(rows * 17 + F)
    ws = vb.varco_ops_workspace(F)
    for residual, gain, quantize in ((True, True, True), (False, False, False), (False, True, True)):
        h, dy, dr = randn(rows, F, g, 2.0), randn(rows, F, g, 1e-2), randn(rows, F, g, 1e-2)
        if rows > 2:
            h[2] = 0
        H, DY, DR = matrix(h, dtype), matrix(dy, dtype, 2), matrix(dr, dtype, 1) if residual else None
        G = 1 + 0.3 * torch.randn(F, generator=g, device=DEV) if gain else None
        h, dy = d64(H, F), d64(DY, F)
        rstd32 = (1 / ((h * h).mean(1) + 1e-6).sqrt()).float()
        rstd = rstd32.double()[:, None]
        out = vb.varco_norm_bwd(DY, H, rstd32, F, gain=G, residual_grad=DR, quantize=quantize, workspace=ws)
        t = dy * G.double() if gain else dy
        dot, mag = (t * h).mean(1, keepdim=True), (t * h).abs().mean(1, keepdim=True)
        res = d64(DR, F) if residual else torch.zeros_like(h)
        dx = rstd * (t - h * rstd ** 2 * dot) + res
        err = 128 * U * (rstd * (t.abs() + h.abs() * rstd ** 2 * mag) + res.abs())
        assert bool(((d64(out.dX, F) - dx).abs() <= err + roundoff(dtype) * dx.abs()).all())
        assert not out.dX[:, F:].any()
        if gain:
            want, size = (dy * h * rstd).sum(0), (dy * h * rstd).abs().sum(0)
            # rows of one lane, teams of a CTA, CTAs: the additions that one value passes
            depth = rows / 148 + 64 + 600 / 32 + 37
            assert bool(((out.dgain.double() - want).abs() <= depth * U * size + 1e-30).all())
        else:
            assert out.dgain is None
        if quantize:
            check_eight(out.dX8, out.scales, dx, err)


def test_norm_backward_against_differences():
    """Directional differences of the forward kernel itself: with a step of 2^-7 the third-order term is below 1e-4 of the
    derivative's terms and fp32 rounding of the loss's terms below 2^-24 / 2^-7 of them."""
    g = gen(11)
    rows, F = 37, 100
    x, r, d = randn(rows, F, g), randn(rows, F, g), randn(rows, F, g)
    w, G, dG = randn(rows, F, g), 1 + 0.2 * torch.randn(F, generator=g, device=DEV), torch.randn(F, generator=g, device=DEV)
    ws = vb.varco_ops_workspace(F)
    M = lambda t: matrix(t, torch.float32)  # noqa: E731
    loss = lambda x, r, G: float((d64(vb.varco_norm_fwd(M(x), F, gain=G, residual=M(r)).Y, F) * w.double()).sum())  # noqa: E731
    f = vb.varco_norm_fwd(M(x), F, gain=G, residual=M(r))
    b = vb.varco_norm_bwd(M(w), f.H, f.rstd, F, gain=G, workspace=ws)
    e = 2.0 ** -7
    size = float(w.abs().double().sum())
    tol = 1e-4 * size + size * U / e
    along = float((d64(b.dX, F) * d.double()).sum())
    assert abs((loss(x + e * d, r, G) - loss(x - e * d, r, G)) / (2 * e) - along) <= tol
    assert abs((loss(x, r + e * d, G) - loss(x, r - e * d, G)) / (2 * e) - along) <= tol
    assert abs((loss(x, r, G + e * dG) - loss(x, r, G - e * dG)) / (2 * e) - float((b.dgain * dG).double().sum())) <= tol


def test_norm_backward_is_reproducible():
    g = gen(12)
    H, DY = matrix(randn(30001, 256, g), torch.bfloat16), matrix(randn(30001, 256, g), torch.bfloat16)
    G, rstd, ws = torch.ones(256, device=DEV), torch.rand(30001, generator=g, device=DEV), vb.varco_ops_workspace(256)
    a, b = (vb.varco_norm_bwd(DY, H, rstd, 256, gain=G, workspace=ws) for _ in range(2))
    assert torch.equal(a.dX, b.dX) and torch.equal(a.dgain, b.dgain)


def test_gain_gradient_calls_in_a_row():
    """Every way of joining the gain gradient (one CTA, the last one, another kernel) in one workspace, without a wait between
    the calls and with the clipped step's barrier in between: each call finds the counters as it left them.  A value passes
    fewer additions than it has rows, so (rows + 2) u of the magnitudes bounds it."""
    g = gen(13)
    ws, some = vb.varco_ops_workspace(1024), [torch.ones(5000, device=DEV)]
    cases = []
    for F in (3, 31, 33, 64, 100, 256, 257, 1000):
        for rows in (1, 2, 31, 33, 130, 500, 2000, 9000):
            for dtype in (torch.float32, torch.bfloat16):
                H, DY = matrix(randn(rows, F, g), dtype), matrix(randn(rows, F, g), dtype)
                rstd = torch.rand(rows, generator=g, device=DEV)
                cases.append((H, DY, rstd, torch.ones(F, device=DEV), F))
    run = lambda c: vb.varco_norm_bwd(c[1], c[0], c[2], c[4], gain=c[3], workspace=ws).dgain  # noqa: E731
    first = []
    for c in cases:
        first.append(run(c))
        norm = vb.varco_grad_norm(some, ws)
    again = [run(c) for c in cases]
    for c, a, b in zip(cases, first, again):
        H, DY, rstd, _, F = c
        terms = d64(H, F) * d64(DY, F) * rstd.double()[:, None]
        assert bool(((a.double() - terms.sum(0)).abs() <= (terms.shape[0] + 2) * U * terms.abs().sum(0) + 1e-30).all()), (F, terms.shape[0])
        assert torch.equal(a, b)
    assert abs(float(norm) - 5000 ** 0.5) <= 4 * U * 5000 ** 0.5
    assert vb.varco_workspace_status(ws) == 0


@pytest.mark.parametrize("most", [445, 602, 640, 1000, 1536])
def test_gain_gradient_in_the_workspace_of_wider_rows(most):
    """A workspace for rows up to `most` wide serves every narrower one, with as many CTAs as the GPU takes.  Values pass fewer
    additions than there are rows."""
    g = gen(most)
    ws = vb.varco_ops_workspace(most)
    for F in (442, 443, 512, 600, most):
        if F <= most:
            H, DY = matrix(randn(20000, F, g), torch.bfloat16), matrix(randn(20000, F, g), torch.bfloat16)
            rstd = torch.rand(20000, generator=g, device=DEV)
            out = vb.varco_norm_bwd(DY, H, rstd, F, gain=torch.ones(F, device=DEV), workspace=ws).dgain
            terms = d64(H, F) * d64(DY, F) * rstd.double()[:, None]
            assert bool(((out.double() - terms.sum(0)).abs() <= 20002 * U * terms.abs().sum(0)).all())


# ------------------------------------------------------------------------------------------ 8-bit forms
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,F", [(1, 1), (2, 128), (7, 129), (1000, 47), (33, 602), (5, 5000)])
def test_quantize_rows(rows, F, dtype):
    g = gen(rows + F)
    x = randn(rows, F, g) * torch.exp(4 * torch.randn((rows, 1), generator=g, device=DEV))
    x[0, 0] = 1e-30
    if rows > 1:
        x[1] = 0
    X = matrix(x, dtype, 1)
    out = vb.varco_quantize_rows(X, F)
    check_eight(out.data, out.scales, d64(X, F), torch.zeros_like(d64(X, F)))
    assert not out.data.view(torch.uint8)[:, F:ld_of(F, dtype)].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("R,K", [(1, 1), (128, 128), (41, 602), (256, 1024), (300, 129), (1000, 77)])
def test_quantize_weight(R, K, dtype):
    g = gen(R * 7 + K)
    W = (torch.randn((R, K + 3), generator=g, device=DEV)).to(dtype)[:, :K]          # rows of any stride
    out = vb.varco_quantize_weight(W)
    w = W.double()
    nr, nk = (R + 127) // 128, (K + 127) // 128
    top = torch.nn.functional.pad(w.abs(), (0, nk * 128 - K, 0, nr * 128 - R)).view(nr, 128, nk, 128).amax((1, 3)) / 448
    assert bool(((out.scales.double() - top).abs() <= 2 * U * top).all())
    s = out.scales.double().repeat_interleave(128, 0)[:R].repeat_interleave(128, 1)[:, :K]
    v = d64(out.data, K) * s
    assert bool(((v - w).abs() <= torch.maximum(w.abs() * 2.0 ** -4, s * 2.0 ** -10) * (1 + 1e-5)).all())
    assert torch.equal(out.data.view(torch.uint8)[:, :K].t().contiguous(), out.transposed.view(torch.uint8)[:, :R].contiguous())
    assert not out.data.view(torch.uint8)[:, K:].any() and not out.transposed.view(torch.uint8)[:, R:].any()


def defined_eight(x, least=2.0 ** -126):
    """(bytes, scales) of rows of 32-bit values by the definition, one IEEE operation after the other."""
    rows, F = x.shape
    nb = (F + 127) // 128
    p = torch.nn.functional.pad(x, (0, nb * 128 - F)).view(rows, nb, 128)
    s = (p.abs().amax(2) * torch.tensor(1 / 448, device=DEV)).clamp_min(least)
    q = (p * (1 / s)[:, :, None]).clamp(-448.0, 448.0).to(E4M3).view(torch.uint8).view(rows, nb * 128)
    return q[:, :F], s.t()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,F", [(3000, 256), (777, 602), (60, 4100)])
def test_eight_bits_are_the_definitions(rows, F, dtype):
    """Bytes and scales bit for bit, over 60 binades and down to the least scale; ties (bf16 rows are full of them) to even."""
    g = gen(rows)
    x = randn(rows, F, g) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=g, device=DEV).float())
    x[:9] *= 2.0 ** -100
    X = matrix(x, dtype)
    x = X[:, :F].float()
    e = vb.varco_quantize_rows(X, F)
    q, s = defined_eight(x)
    assert torch.equal(e.scales, s) and torch.equal(e.data.view(torch.uint8)[:, :F], q)
    w = vb.varco_quantize_weight(X[:, :F])
    nr, nk = (rows + 127) // 128, (F + 127) // 128
    p = torch.nn.functional.pad(x, (0, nk * 128 - F, 0, nr * 128 - rows)).view(nr, 128, nk, 128)
    s = (p.abs().amax((1, 3)) * torch.tensor(1 / 448, device=DEV)).clamp_min(2.0 ** -126)
    q = (p * (1 / s)[:, None, :, None]).clamp(-448.0, 448.0).to(E4M3).view(torch.uint8).view(nr * 128, nk * 128)[:rows, :F]
    assert torch.equal(w.scales, s) and torch.equal(w.data.view(torch.uint8)[:, :F], q)
    assert torch.equal(w.transposed.view(torch.uint8)[:, :rows], q.t())
    if dtype == torch.float32:                            # the norm's and the product's outputs in 32 bits are what they quantise
        n = vb.varco_norm_fwd(X, F, quantize=True)
        q, s = defined_eight(n.Y[:, :F].contiguous())
        assert torch.equal(n.scales, s) and torch.equal(n.Y8.view(torch.uint8)[:, :F], q)
        B, _ = weight(F, F, g)
        for M in (20, rows):
            out = vb.varco_fp8_product(e.data[:M], e.scales[:, :M], B.data, B.scales, F, dtype=dtype, quantize=True, workspace=vb.varco_ops_workspace())
            q, s = defined_eight(out.Y[:, :F].contiguous())
            assert torch.equal(out.scales, s) and torch.equal(out.Y8.view(torch.uint8)[:, :F], q)


# ------------------------------------------------------------------------------------------ product
def operand(rows, F, g, extra=0, scale=1.0):
    """8-bit matrix with row-block scales whose padding bytes are NaN, its scales with a row stride of their own."""
    x = randn(rows, F, g, scale)
    if rows > 3:
        x[2] = 0
    e = vb.varco_quantize_rows(matrix(x, torch.float32), F)
    m = torch.full((rows, ld_of(F, E4M3, extra)), 0x7F, dtype=torch.uint8, device=DEV)
    m[:, :F] = e.data.view(torch.uint8)[:, :F]
    s = torch.full((e.scales.shape[0], rows + 5), float("nan"), device=DEV)
    s[:, :rows] = e.scales
    m = m.view(E4M3)
    return m, s[:, :rows], d64(m, F) * spread(e.scales, F)


def weight(N, K, g):
    e = vb.varco_quantize_weight(torch.randn((N, K), generator=g, device=DEV) / K ** 0.5)
    s = e.scales.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    return e, d64(e.data, K) * s


def product_error(a, b, K):
    return 2.0 ** -22 * (K / 32 + K / 128 + 4) * (a.abs() @ b.abs().t())


SHAPES = [(1, 1, 1), (1, 256, 256), (5, 1024, 256), (16, 41, 602), (17, 64, 100), (33, 47, 256), (128, 128, 128), (129, 129, 129),
          (200, 300, 500), (1000, 256, 1024), (130, 1024, 2048), (3, 520, 4096), (260, 513, 1300), (8, 2048, 130), (2, 16, 8200),
          (4000, 256, 256), (40001, 256, 128)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_fp8_product(M, N, K, dtype):
    g = gen(M + 3 * N + 7 * K)
    ws = vb.varco_ops_workspace()
    A8, sA, a = operand(M, K, g, 1)
    B, b = weight(N, K, g)
    acc, err = a @ b.t(), product_error(a, b, K)
    for bias, relu, masked, keep, quantize in ((True, True, False, True, True), (False, False, False, True, False),
                                               (False, False, True, True, True), (True, False, False, False, True)):
        c = torch.randn(N, generator=g, device=DEV) if bias else None
        mask = None
        if masked:
            u = randn(M, N, g)
            u[0, 0] = float("nan")                   # not positive
            mask = matrix(u, dtype, 1)
        out = vb.varco_fp8_product(A8, sA, B.data, B.scales, K, bias=c, relu=relu, mask=mask, dtype=dtype, keep=keep, quantize=quantize,
                                   workspace=ws)
        y = acc + c.double() if bias else acc
        e = err + 2 * U * y.abs()
        if relu:
            y = y.clamp_min(0)
        if masked:
            on = mask[:, :N] > 0
            y, e = torch.where(on, y, 0.0), torch.where(on, e, 0.0)
        if keep:
            assert bool(((d64(out.Y, N) - y).abs() <= e + roundoff(dtype) * y.abs()).all())
        else:
            assert out.Y is None
        if quantize:
            check_eight(out.Y8, out.scales, y, e)
    assert vb.varco_workspace_status(ws) == 0


@pytest.mark.parametrize("M,N,K", [(9, 300, 700), (18, 41, 602), (24, 1024, 1024), (25, 129, 257), (31, 513, 1300), (32, 4096, 130),
                                   (32, 16, 4096), (7, 9600, 64), (17, 4800, 200), (8, 9600, 1030)])
def test_fp8_product_few_rows(M, N, K):
    """Both sides of the places where the form for few rows ends: 8, 16, 24 and 32 rows, widths at which its CTAs no longer
    run all at once."""
    test_fp8_product(M, N, K, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(20001, 100, 300), (40000, 128, 700), (19000, 65, 1300), (12001, 700, 1300), (5000, 513, 602), (9700, 256, 2100),
                                   (19100, 1025, 140), (40001, 41, 602), (60000, 64, 1000), (38000, 1, 129), (1500, 900, 1100), (37, 3000, 520)])
def test_fp8_product_many_tiles_and_blocks(M, N, K, dtype):
    """Every tile form by value where a CTA works through several tiles of several blocks: accumulators in turn, operand stages
    that wrap inside a tile, scales that change along K and from tile to tile, outputs that are ragged both ways.  Two CTAs of 128
    columns (N of 65 to 128, more row tiles than SMs), one of 256, two of 64, one of 128."""
    test_fp8_product(M, N, K, dtype)


def test_fp8_product_values_repeat():
    """Calls in a row give the same bits, and these are right."""
    g = gen(26)
    ws = vb.varco_ops_workspace()
    for M, N, K in ((20001, 100, 700), (5000, 500, 700), (30000, 41, 300)):
        A8, sA, a = operand(M, K, g)
        B, b = weight(N, K, g)
        outs = [vb.varco_fp8_product(A8, sA, B.data, B.scales, K, quantize=True, workspace=ws) for _ in range(5)]
        y = a @ b.t()
        e = product_error(a, b, K) + 2 * U * y.abs()
        assert bool(((d64(outs[0].Y, N) - y).abs() <= e + 2.0 ** -8 * y.abs()).all())
        check_eight(outs[0].Y8, outs[0].scales, y, e)
        for o in outs[1:]:
            assert torch.equal(o.Y[:, :N], outs[0].Y[:, :N]) and torch.equal(o.scales, outs[0].scales)
            assert torch.equal(o.Y8.view(torch.uint8)[:, :N], outs[0].Y8.view(torch.uint8)[:, :N])


def test_few_rows_clusters_that_start_apart():
    """The CTAs of a cluster exchange their rows' largest magnitudes.  Widths that leave a cluster's last CTAs without columns and
    more clusters than run at once, launched back to back: every call gives the first one's scales and bytes, and these are right."""
    g = gen(25)
    ws = vb.varco_ops_workspace()
    for M, N, K in ((1, 9400, 128), (8, 9400, 1100), (8, 8288, 64), (8, 8289, 64), (8, 4096, 64), (20, 1040, 3000), (32, 4144, 64),
                    (32, 4145, 64), (32, 130, 16), (5, 17, 1)):
        A8, sA, a = operand(M, K, g)
        B, b = weight(N, K, g)
        outs = [vb.varco_fp8_product(A8, sA, B.data, B.scales, K, keep=False, quantize=True, workspace=ws) for _ in range(40)]
        y = a @ b.t()
        check_eight(outs[0].Y8, outs[0].scales, y, product_error(a, b, K) + 2 * U * y.abs())
        for o in outs[1:]:
            assert torch.equal(o.scales, outs[0].scales)
            assert torch.equal(o.Y8.view(torch.uint8)[:, :N], outs[0].Y8.view(torch.uint8)[:, :N])


def test_fp8_product_backward_is_the_adjoint():
    """<dY, A B^T> = <dY B, A> with the 8-bit forms of both sides: the transposed bytes and exchanged scale strides of a
    weight are the same matrix."""
    g = gen(21)
    M, N, K = 700, 300, 520
    ws = vb.varco_ops_workspace()
    A8, sA, a = operand(M, K, g)
    D8, sD, d = operand(M, N, g, scale=1e-3)
    B, b = weight(N, K, g)
    y = vb.varco_fp8_product(A8, sA, B.data, B.scales, K, dtype=torch.float32, workspace=ws).Y
    da = vb.varco_fp8_product(D8, sD, B.transposed, B.scales.t(), N, dtype=torch.float32, workspace=ws).Y
    left, right = (d64(y, N) * d).sum(), (d64(da, K) * a).sum()
    tol = (product_error(a, b, K) * d.abs()).sum() + (product_error(d, b.t(), N) * a.abs()).sum()
    assert abs(float(left - right)) <= float(tol)


def test_fp8_product_infinite_and_nan_rows_stay_in_their_rows():
    g = gen(22)
    ws = vb.varco_ops_workspace()
    x = randn(40, 256, g)
    x[3, 5], x[20, 200] = float("nan"), float("inf")
    e = vb.varco_quantize_rows(matrix(x, torch.float32), 256)
    B, _ = weight(200, 256, g)
    out = vb.varco_fp8_product(e.data, e.scales, B.data, B.scales, 256, relu=True, quantize=True, workspace=ws)
    bad = torch.zeros(40, dtype=torch.bool, device=DEV)
    bad[[3, 20]] = True
    assert bool(torch.isfinite(out.Y[~bad]).all()) and bool(torch.isfinite(out.scales[:, ~bad]).all())
    assert bool(torch.isnan(out.Y[bad][:, :200].float()).all()) and bool(torch.isnan(out.scales[:, bad]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(5, 41, 130), (30, 200, 64), (40, 41, 130), (40, 100, 64), (200, 70, 300), (40, 200, 64), (1000, 300, 64),
                                   (20001, 100, 130), (9001, 531, 130)])
def test_masked_rows_that_are_not_finite(M, N, K, dtype):
    """A row of A with a NaN and one with an infinity, masked whole and in part: what the mask leaves out is zero, in both outputs,
    whatever stands there; a mask's padding (here ones) is no mask.  All other rows are as without them."""
    g = gen(M + N)
    ws = vb.varco_ops_workspace()
    x = randn(M, K, g)
    x[1, 0], x[2, K - 1], x[3, 1], x[4, 2] = float("nan"), float("inf"), float("nan"), -float("inf")
    A = vb.varco_quantize_rows(matrix(x, torch.float32), K)
    B, b = weight(N, K, g)
    u = randn(M, N, g)
    u[1:3] = 0                                           # nothing is left of rows 1 and 2
    u[3, :N - 1], u[3, N - 1] = -1, 1                    # the last column is left of row 3
    out = vb.varco_fp8_product(A.data, A.scales, B.data, B.scales, K, mask=matrix(u, dtype, 1, fill=1.0), dtype=dtype, quantize=True,
                               workspace=ws)
    bad = [1, 2, 3, 4]
    last = (N - 1) // 128 * 128                          # first column of the last block
    assert not out.Y[1:3, :N].any() and not out.Y8[1:3, :N].view(torch.uint8).any()
    assert bool((out.scales[:, 1:3] == 2.0 ** -126).all())
    assert not out.Y[3, :N - 1].any() and bool(torch.isnan(out.Y[3, N - 1]))
    v = out.Y8[:, :N].double() * spread(out.scales, N)
    assert not v[3, :last].any() and bool(torch.isnan(v[3, last:N]).all())
    good = torch.ones(M, dtype=torch.bool, device=DEV)
    good[bad] = False
    a = A.data[good].double()[:, :K] * spread(A.scales[:, good].contiguous(), K)
    on = u.to(dtype)[good] > 0
    y, e = torch.where(on, a @ b.t(), 0.0), torch.where(on, product_error(a, b, K) + 2 * U * (a @ b.t()).abs(), 0.0)
    assert bool(((d64(out.Y[good], N) - y).abs() <= e + roundoff(dtype) * y.abs()).all())
    check_eight(out.Y8[good], out.scales[:, good].contiguous(), y, e)


def test_fp8_product_is_reproducible_and_empty():
    g = gen(23)
    ws = vb.varco_ops_workspace()
    A8, sA, _ = operand(5000, 700, g)
    B, _ = weight(500, 700, g)
    one, two = (vb.varco_fp8_product(A8, sA, B.data, B.scales, 700, workspace=ws).Y for _ in range(2))
    assert torch.equal(one[:, :500], two[:, :500])
    out = vb.varco_fp8_product(A8[:0], sA[:, :0], B.data, B.scales, 700, quantize=True, workspace=ws)
    assert out.Y.shape[0] == 0 and out.scales.shape == (4, 0)


def test_product_on_another_stream():
    """Operands made on the default stream, the call on a side stream that waits for them."""
    g = gen(24)
    ws = vb.varco_ops_workspace()
    A8, sA, a = operand(900, 256, g)
    B, b = weight(256, 256, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = vb.varco_fp8_product(A8, sA, B.data, B.scales, 256, dtype=torch.float32, workspace=ws).Y
    torch.cuda.current_stream().wait_stream(side)
    assert bool(((d64(y, 256) - a @ b.t()).abs() <= product_error(a, b, 256) + 2 * U * (a @ b.t()).abs()).all())


# ------------------------------------------------------------------------------------------ weight gradient
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,Fa,Fb", [(0, 5, 9), (1, 8, 8), (100, 256, 64), (777, 47, 602), (3000, 1024, 256), (500, 1100, 300)])
def test_weight_grad(rows, Fa, Fb, dtype):
    g = gen(rows + Fa)
    A, B = matrix(randn(rows, Fa, g), dtype), matrix(randn(rows, Fb, g), dtype)
    ws = vb.varco_weight_grad_workspace(Fa, Fb)
    dW, db = vb.varco_weight_grad(A, Fa, B, Fb, ws)
    a, b = d64(A, Fa), d64(B, Fb)
    # every product and every addition rounds once: rows + 1 roundings of the magnitudes cover any order of them
    assert bool(((dW.double() - a.t() @ b).abs() <= 2 * (rows + 1) * U * (a.abs().t() @ b.abs()) + 1e-30).all())
    assert bool(((db.double() - a.sum(0)).abs() <= (rows + 1) * U * a.abs().sum(0) + 1e-30).all())
    assert vb.varco_workspace_status(ws) == 0


# ------------------------------------------------------------------------------------------ padding of outputs
def garbage(rows, ld, dtype):
    return torch.full((rows, ld * torch.empty((), dtype=dtype).element_size()), 0x7F, dtype=torch.uint8, device=DEV).view(dtype)


def check_padding(t, F):
    """Zero from column F to the next 16 bytes, untouched from there."""
    es = t.element_size()
    b, end = t.view(torch.uint8), ld_of(F, t.dtype) * es
    assert not b[:, F * es:end].any() and bool((b[:, end:] == 0x7F).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("F", [1, 3, 4, 5, 8, 9, 15, 16, 17, 20, 127, 129, 300, 602, 1001, 4100])
def test_padding_of_outputs(F, dtype):
    """Outputs wider than their rows, full of bytes that are neither zero nor finite e4m3 values, at the C ABI; among the rows a
    NaN and an infinity, whose scales are not finite."""
    g, L, st = gen(F), vb.lib(), torch.cuda.current_stream().cuda_stream
    dt, rows = vb.F32 if dtype == torch.float32 else vb.BF16, 37
    x = randn(rows, F, g)
    x[3, 0], x[5, F - 1] = float("nan"), float("inf")
    X = matrix(x, dtype)
    G, ws = torch.ones(F, device=DEV), vb.varco_ops_workspace(F)
    P = lambda t: t.data_ptr()  # noqa: E731
    ld, ld8, nb = ld_of(F, dtype, 3), ld_of(F, E4M3, 3), (F + 127) // 128
    H, Y, Y8 = garbage(rows, ld, dtype), garbage(rows, ld, dtype), garbage(rows, ld8, E4M3)
    s, rstd, dg = torch.empty((nb, rows), device=DEV), torch.empty(rows, device=DEV), torch.empty(F, device=DEV)
    d = vb.NormDesc(rows, F, dt, 1e-6, X.shape[1], X.shape[1], ld, ld, ld8, rows)
    assert L.varco_norm_fwd(d, P(X), P(X), P(G), P(H), P(Y), P(Y8), P(s), P(rstd), st) == 0
    for t in (H, Y, Y8):
        check_padding(t, F)
    dX, dX8 = garbage(rows, ld, dtype), garbage(rows, ld8, E4M3)
    d = vb.NormDesc(rows, F, dt, 1e-6, ld, X.shape[1], X.shape[1], X.shape[1], ld8, rows)
    assert L.varco_norm_bwd(d, P(X), P(X), P(rstd), P(G), P(X), P(dX), P(dX8), P(s), P(dg), P(ws), ws.numel(), st) == 0
    check_padding(dX, F), check_padding(dX8, F)
    Y8 = garbage(rows, ld8, E4M3)
    assert L.varco_quantize_rows(rows, F, dt, P(X), X.shape[1], P(Y8), ld8, P(s), rows, st) == 0
    check_padding(Y8, F)
    W8, T8, sw = garbage(rows, ld8, E4M3), garbage(F, ld_of(rows, E4M3, 20), E4M3), torch.empty((1, nb), device=DEV)
    assert L.varco_quantize_weight(rows, F, dt, P(X), X.shape[1], P(W8), ld8, P(T8), T8.shape[1], P(sw), nb, st) == 0
    check_padding(W8, F), check_padding(T8, rows)
    # products of few rows and of many (tiles), F columns out: the weight's transposed bytes, 37 in use, as B
    B, b = weight(F, rows, g)
    for M in (1, 7, 30, 37, 300):
        a = randn(M, rows, g)
        a[M // 2, 0] = float("nan")
        A = vb.varco_quantize_rows(matrix(a, torch.float32), rows)
        Y, Y8, s = garbage(M, ld, dtype), garbage(M, ld8, E4M3), torch.empty((nb, M), device=DEV)
        c = torch.randn(F, generator=g, device=DEV)
        d = vb.Fp8Desc(M, F, rows, dt, 0, A.data.shape[1], B.data.shape[1], M, 1, 1, 0, ld, ld8, M)
        assert L.varco_fp8_product(d, P(A.data), P(A.scales), P(B.data), P(B.scales), P(c), 0, P(Y), P(Y8), P(s), P(ws), ws.numel(), st) == 0
        check_padding(Y, F), check_padding(Y8, F)
        Y = garbage(M, ld, dtype)
        assert L.varco_fp8_product(d, P(A.data), P(A.scales), P(B.data), P(B.scales), P(c), 0, P(Y), 0, 0, P(ws), ws.numel(), st) == 0
        check_padding(Y, F)


# ------------------------------------------------------------------------------------------ slices of rows
@pytest.mark.parametrize("n", [1, 2, 5])
def test_slices_of_padded_matrices_with_any_number_of_rows(n):
    """The first n rows and the columns in use of padded matrices, as a caller slices them: one row is taken as several are, and
    gives what it gives among them."""
    g = gen(31)
    ws, gws, G = vb.varco_ops_workspace(60), vb.varco_weight_grad_workspace(60, 60), torch.ones(60, device=DEV)
    cut = lambda t, F=60: t[:n, :F]  # noqa: E731
    same = lambda a, b, F=60: torch.equal(a[:, :F].contiguous().view(torch.uint8), b[:n, :F].contiguous().view(torch.uint8))  # noqa: E731
    M = matrix(randn(5, 60, g), torch.bfloat16)
    all_, some = (vb.varco_norm_fwd(x, 60, gain=G, residual=x, quantize=True) for x in (M, cut(M)))
    assert same(some.Y, all_.Y) and same(some.H, all_.H) and same(some.Y8, all_.Y8) and torch.equal(some.scales, all_.scales[:, :n])
    back = [vb.varco_norm_bwd(f(M), f(all_.H), f(all_.rstd[:, None], 1)[:, 0].contiguous(), 60, gain=G, residual_grad=f(M), workspace=ws).dX
            for f in (lambda t, F=60: t, cut)]
    assert same(back[1], back[0])
    e = vb.varco_quantize_rows(cut(M), 60)
    W = vb.varco_quantize_weight(torch.randn((20, 60), generator=g, device=DEV))
    mask = matrix(randn(5, 20, g), torch.bfloat16)
    p = [vb.varco_fp8_product(f(a), s, W.data[:, :60], W.scales, 60, mask=f(mask, 20), workspace=ws).Y
         for f, a, s in ((lambda t, F=60: t[:, :F], vb.varco_quantize_rows(M, 60).data, vb.varco_quantize_rows(M, 60).scales), (cut, e.data, e.scales))]
    assert same(p[1], p[0], 20)
    dW, _ = vb.varco_weight_grad(cut(M), 60, cut(M), 60, gws)
    a = d64(M, 60)[:n]
    assert bool(((dW.double() - a.t() @ a).abs() <= 2 * (n + 1) * U * (a.abs().t() @ a.abs())).all())


def test_a_single_row_that_ends_with_its_columns_is_refused_as_several_are():
    for n in (1, 2):
        with pytest.raises(vb.VarcoError):
            vb.varco_norm_fwd(torch.zeros((n, 60), dtype=torch.bfloat16, device=DEV), 60)


# ------------------------------------------------------------------------------------------ graphs
@pytest.mark.parametrize("rows", [5, 3000])
def test_every_call_in_a_graph(rows):
    """Calls captured in a CUDA graph, replayed on new inputs in the same buffers: what the calls themselves give for these."""
    g = gen(rows)
    width, hidden, dt = 300, 700, torch.bfloat16
    ws, gws = vb.varco_ops_workspace(width), vb.varco_weight_grad_workspace(hidden, width)
    X, R, G = matrix(randn(rows, width, g), dt), matrix(randn(rows, width, g), dt), torch.rand(width, generator=g, device=DEV) + 0.5
    W = randn(hidden, width, g, 0.05)
    P, C = W.clone(), W.bfloat16()

    def step():
        n = vb.varco_norm_fwd(X, width, gain=G, residual=R, quantize=True)
        q = vb.varco_quantize_weight(W)
        u = vb.varco_fp8_product(n.Y8, n.scales, q.data, q.scales, width, relu=True, quantize=True, workspace=ws)
        d = vb.varco_fp8_product(u.Y8, u.scales, q.transposed, q.scales.t(), hidden, workspace=ws)
        b = vb.varco_norm_bwd(d.Y, n.H, n.rstd, width, gain=G, residual_grad=R, quantize=True, workspace=ws)
        dW, db = vb.varco_weight_grad(u.Y, hidden, n.Y, width, gws)
        e = vb.varco_quantize_rows(b.dX, width)
        norm = vb.varco_grad_norm([dW, db], ws)
        vb.varco_clip_step([P], [dW], 0.1, 1.0, copies=[C], workspace=ws)
        vb.varco_grad_clip([db], 0.5, ws)
        return [n.Y8.view(torch.uint8)[:, :width], u.Y[:, :hidden], u.scales, b.dX[:, :width], b.dgain, dW, db, e.scales, norm, P, C]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            out = step()
    torch.cuda.synchronize()
    for seed in (1, 2):
        X[:, :width] = randn(rows, width, gen(seed)).to(dt)
        P.copy_(W), C.copy_(W)
        graph.replay()
        got = [t.clone() for t in out]
        P.copy_(W), C.copy_(W)
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
    assert vb.varco_workspace_status(ws) == 0 and vb.varco_workspace_status(gws) == 0


# ------------------------------------------------------------------------------------------ refusals
def test_refusals():
    X = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    ws = vb.varco_ops_workspace(64)
    G = torch.ones(64, device=DEV)
    bad = pytest.raises((ValueError, TypeError, vb.VarcoError))
    with bad:
        vb.varco_norm_fwd(X.half(), 64)                                   # type
    with bad:
        vb.varco_norm_fwd(X, 65)                                          # more columns than there are
    with bad:
        vb.varco_norm_fwd(X[:, 1:], 60)                                   # base not aligned
    with bad:
        vb.varco_norm_fwd(X.t(), 4)                                       # rows not contiguous
    with bad:
        vb.varco_norm_fwd(X[:, :60].contiguous(), 60)                     # row stride no multiple of 16 bytes
    with bad:
        vb.varco_norm_fwd(X, 64, residual=X[:3])
    with bad:
        vb.varco_norm_fwd(X, 64, residual=X.float())
    with bad:
        vb.varco_norm_fwd(X, 64, gain=G.bfloat16())
    with bad:
        vb.varco_norm_fwd(X, 64, gain=G[:63])
    with bad:
        vb.varco_norm_fwd(X, 64, eps=0.0)
    with bad:
        vb.varco_norm_fwd(torch.zeros((1, 20000), device=DEV), 20000)     # wider than the kernels cover
    with bad:
        vb.varco_norm_bwd(X, X, torch.zeros(4, device=DEV), 64, gain=G)   # no workspace
    with bad:
        vb.varco_norm_bwd(X, X, torch.zeros(4, device=DEV), 64, gain=G, workspace=ws[:1000])
    e = vb.varco_quantize_rows(X, 64)
    W = vb.varco_quantize_weight(torch.zeros((32, 64), device=DEV))
    ok = dict(workspace=ws)
    vb.varco_fp8_product(e.data, e.scales, W.data, W.scales, 64, **ok)
    with bad:
        vb.varco_fp8_product(X, e.scales, W.data, W.scales, 64, **ok)
    with bad:
        vb.varco_fp8_product(e.data, e.scales[:, :3], W.data, W.scales, 64, **ok)
    with bad:
        vb.varco_fp8_product(e.data, e.scales, W.data, W.scales.double(), 64, **ok)
    with bad:
        vb.varco_fp8_product(e.data, e.scales, W.data, W.scales[:0], 64, **ok)
    with bad:
        vb.varco_fp8_product(e.data, e.scales, W.data, W.scales, 128, **ok)
    with bad:
        vb.varco_fp8_product(e.data, e.scales, W.data, W.scales, 64, bias=torch.zeros(31, device=DEV), **ok)
    with bad:
        vb.varco_fp8_product(e.data, e.scales, W.data, W.scales, 64, mask=torch.zeros((4, 32), device=DEV), **ok)   # not of dtype
    with bad:
        vb.varco_fp8_product(e.data, e.scales, W.data, W.scales, 64, dtype=torch.float16, **ok)
    with bad:
        vb.varco_fp8_product(e.data, e.scales, W.data, W.scales, 64, keep=False, **ok)                             # no output
    with bad:
        vb.varco_fp8_product(e.data, e.scales, W.data, W.scales, 64)                                               # no workspace
    with bad:
        vb.varco_quantize_weight(torch.zeros((32, 64), device=DEV).t())
    assert vb.varco_workspace_status(ws) == 0
