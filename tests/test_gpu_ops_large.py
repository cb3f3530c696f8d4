"""Offsets past 2^31 elements: rows near both ends of large matrices against 64 bits (bounds as in the small tests)."""
import pytest
import torch

from paper_2406_17611_b200 import binding as vb

from test_gpu_ops import U, check_eight, d64, gen, matrix, product_error, spread, weight

pytestmark = pytest.mark.gpu

ROWS, F = 2_200_003, 1000            # 2.2e9 elements


def test_product_and_norm_past_31_bits():
    g = gen(1)
    ws = vb.varco_ops_workspace(F)
    x = torch.randn((ROWS, 128), generator=g, device="cuda:0").bfloat16()
    A = vb.varco_quantize_rows(x, 128)
    B, b = weight(F, 128, g)
    out = vb.varco_fp8_product(A.data, A.scales, B.data, B.scales, 128, quantize=True, workspace=ws)
    ends = torch.cat([torch.arange(300), torch.arange(ROWS // 2, ROWS // 2 + 300), torch.arange(ROWS - 300, ROWS)]).cuda()
    a = A.data[ends].double() * spread(A.scales[:, ends].contiguous(), 128)
    y, e = a @ b.t(), product_error(a, b, 128) + 2 * U * (a @ b.t()).abs()
    assert bool(((d64(out.Y[ends], F) - y).abs() <= e + 2.0 ** -8 * y.abs()).all())
    check_eight(out.Y8[ends], out.scales[:, ends].contiguous(), y, e)
    # masked with itself: only what is positive stays, read from the same far rows
    back = vb.varco_fp8_product(A.data, A.scales, B.data, B.scales, 128, mask=out.Y, workspace=ws).Y[ends]
    on = out.Y[ends][:, :F] > 0
    assert torch.equal(back[:, :F], torch.where(on, out.Y[ends][:, :F], 0.0))
    del back
    n = vb.varco_norm_fwd(out.Y, F, quantize=True)
    h = d64(out.Y[ends], F)
    want = h / ((h * h).mean(1, keepdim=True) + 1e-6).sqrt()
    assert bool(((d64(n.Y[ends], F) - want).abs() <= (128 * U + 2.0 ** -8) * want.abs()).all())
    check_eight(n.Y8[ends], n.scales[:, ends].contiguous(), want, 128 * U * want.abs())
    r = vb.varco_norm_bwd(n.Y, out.Y, n.rstd, F)
    t, s = d64(n.Y[ends], F), n.rstd[ends].double()[:, None]
    d = s * (t - h * s * s * (t * h).mean(1, keepdim=True))
    m = s * (t.abs() + h.abs() * s * s * (t * h).abs().mean(1, keepdim=True))
    assert bool(((d64(r.dX[ends], F) - d).abs() <= 128 * U * m + 2.0 ** -8 * d.abs()).all())
    assert vb.varco_workspace_status(ws) == 0
    # one tensor of that size in the clipped step
    w = torch.ones(ROWS * F, device="cuda:0")
    del out, n, r
    gr = torch.full((ROWS * F,), 0.5, device="cuda:0")
    gr[-1] = 4.0
    norm = vb.varco_clip_step([w], [gr], 1.0, 1e30, workspace=ws)
    assert abs(float(norm) - (0.25 * (ROWS * F - 1) + 16.0) ** 0.5) <= 2.0 ** -20 * float(norm)
    assert float(w[0]) == 0.5 and float(w[-1]) == -3.0 and float(w[-2]) == 0.5 and float(w[ROWS * F // 2]) == 0.5


def test_product_of_more_than_two_gigabytes_a_row():
    """One row of 600 million columns in fp32 with mask and 8-bit output: byte offsets inside the row pass 2^31, scale strides
    too.  The columns around 2^29, where a 32-bit byte offset wraps, and both ends against 64 bits."""
    N, K = 600_000_000, 16
    g = gen(2)
    ws = vb.varco_ops_workspace()
    A = vb.varco_quantize_rows(torch.randn((1, K), generator=g, device="cuda:0"), K)
    B = torch.randint(0, 0x7F, (N, K), generator=g, device="cuda:0", dtype=torch.uint8).view(torch.float8_e4m3fn)     # 0 to 448
    sB = torch.rand(((N + 127) // 128, 1), generator=g, device="cuda:0") + 0.5
    mask = torch.randn((1, N), generator=g, device="cuda:0")
    out = vb.varco_fp8_product(A.data, A.scales, B, sB, K, mask=mask, dtype=torch.float32, quantize=True, workspace=ws)
    assert vb.varco_workspace_status(ws) == 0
    a = A.data.double() * A.scales.double()
    for at in (0, (1 << 28) - 512, (1 << 29) - 512, (1 << 29) + 128 * 9999, N - N % 128 - 1024):
        cols = torch.arange(at, min(at + 1024, N), device="cuda:0")
        b = B[cols].double() * sB[cols // 128].double()
        on = mask[:, cols] > 0
        y = torch.where(on, a @ b.t(), 0.0)
        e = torch.where(on, product_error(a, b, K) + 2 * U * y.abs(), 0.0)
        assert bool(((out.Y[:, cols].double() - y).abs() <= e + 2 * U * y.abs()).all()), at
        check_eight(out.Y8[:, cols], out.scales[at // 128:(int(cols[-1]) + 128) // 128].contiguous(), y, e)
