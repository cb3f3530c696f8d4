"""Refusals of the residual block's entry points at the C ABI: every bad argument is a status code before anything is
launched, so these run without a GPU (the addresses are never followed)."""
import ctypes as C

import pytest

from paper_2406_17611_b200 import binding as vb
from paper_2406_17611_b200 import build as vbuild

A = 1 << 20            # a 16-byte aligned address that nothing follows
OK, INVALID, TOO_SMALL, UNSUPPORTED = 0, -1, -6, -7


@pytest.fixture(scope="module", autouse=True)
def built():
    vbuild.build()


def norm(**k):
    d = dict(rows=4, F=60, dtype=1, eps=1e-6, ldx=64, ldr=64, ldh=64, ldy=64, ld8=64, lds=4)
    d.update(k)
    return vb.NormDesc(*[d[f] for f, _ in vb.NormDesc._fields_])


def fp8(**k):
    d = dict(M=4, N=32, K=60, dtype=1, relu=0, lda=64, ldb=64, ld_sa=4, sb_n=1, sb_k=1, ldmask=32, ldy=32, ldy8=32, ld_sy=4)
    d.update(k)
    return vb.Fp8Desc(*[d[f] for f, _ in vb.Fp8Desc._fields_])


def test_workspace_sizes():
    b = C.c_size_t()
    L = vb.lib()
    sizes = []
    for F in (1, 256, 4096, 16384):
        assert L.varco_ops_workspace_bytes(F, C.byref(b)) == OK
        sizes.append(b.value)
    assert sizes[0] >= 1184 * 21 * 8 and sizes[-1] >= 148 * 2 * 16384 * 4
    assert L.varco_ops_workspace_bytes(0, C.byref(b)) == INVALID
    assert L.varco_ops_workspace_bytes(16385, C.byref(b)) == UNSUPPORTED
    assert L.varco_weight_grad_workspace_bytes(100, 256, C.byref(b)) == OK and b.value > 512
    assert L.varco_weight_grad_workspace_bytes(0, 256, C.byref(b)) == INVALID


def test_workspace_covers_every_narrower_width():
    """What is sized for F_max is passed with every width up to it, and a call at width F is content with the size for F."""
    b = C.c_size_t()
    L = vb.lib()
    before = 0
    for F in range(1, 16385):
        assert L.varco_ops_workspace_bytes(F, C.byref(b)) == OK
        assert b.value >= before, F
        before = b.value
    # the largest partials of the gain gradient: 4736 lines while they fit 8 MB, then as many lines as do, at least 296
    assert L.varco_ops_workspace_bytes(602, C.byref(b)) == OK and b.value >= 512 + (8 << 20)
    assert L.varco_ops_workspace_bytes(16384, C.byref(b)) == OK and b.value == 512 + 296 * 16384 * 4


@pytest.mark.parametrize("change,want", [
    (dict(rows=-1), INVALID), (dict(F=0), INVALID), (dict(dtype=2), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(F=16385), UNSUPPORTED), (dict(ldx=56), INVALID), (dict(ldx=65), INVALID), (dict(ldy=59), INVALID), (dict(lds=3), INVALID),
    (dict(ld8=60), INVALID), (dict(rows=0), OK)])
def test_norm_forward_arguments(change, want):
    assert vb.lib().varco_norm_fwd(norm(**change), A, A, 0, A, A, A, A, A, 0) == want


def test_norm_pointers():
    L = vb.lib()
    f, b = L.varco_norm_fwd, L.varco_norm_bwd
    assert f(None, A, 0, 0, 0, A, 0, 0, 0, 0) == INVALID
    assert f(norm(), 0, 0, 0, 0, A, 0, 0, 0, 0) == INVALID                 # no input
    assert f(norm(), A + 8, 0, 0, 0, A, 0, 0, 0, 0) == INVALID             # not aligned
    assert f(norm(), A, 0, 0, 0, 0, 0, 0, 0, 0) == INVALID                 # no output
    assert f(norm(), A, 0, 0, 0, A, A, 0, 0, 0) == INVALID                 # 8 bits without scales
    assert f(norm(), A, 0, 0, 0, A, 0, A, 0, 0) == INVALID                 # scales without 8 bits
    assert b(norm(), A, A, 0, 0, 0, A, 0, 0, 0, 0, 0, 0) == INVALID        # no rstd
    assert b(norm(), A, A, A, A, 0, A, 0, 0, A, 0, 0, 0) == INVALID        # gain gradient without a workspace
    assert b(norm(), A, A, A, A, 0, A, 0, 0, A, A, 4096, 0) == TOO_SMALL
    assert b(norm(), A, A, A, 0, 0, 0, 0, 0, 0, 0, 0, 0) == INVALID        # no output
    assert b(norm(rows=0), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0) == OK


@pytest.mark.parametrize("change,want", [
    (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(dtype=7), INVALID), (dict(lda=60), INVALID), (dict(lda=48), INVALID),
    (dict(ldb=72), INVALID), (dict(ld_sa=3), INVALID), (dict(sb_n=-1), INVALID), (dict(ldy=24), INVALID), (dict(ldy=36), INVALID),
    (dict(ldy8=16), INVALID), (dict(ld_sy=2), INVALID), (dict(ldmask=31), INVALID), (dict(M=1 << 31), UNSUPPORTED), (dict(M=0), OK)])
def test_product_arguments(change, want):
    assert vb.lib().varco_fp8_product(fp8(**change), A, A, A, A, A, A, A, A, A, A, 1 << 20, 0) == want


def test_product_pointers():
    f = vb.lib().varco_fp8_product
    ok = [fp8(), A, A, A, A, 0, 0, A, 0, 0, A, 1 << 20, 0]
    for i, v in ((0, None), (1, 0), (1, A + 4), (2, 0), (3, 0), (4, 0), (7, 0), (7, A + 8), (10, 0)):
        args = list(ok)
        args[i] = v
        assert f(*args) == INVALID, i
    assert f(*ok[:8], A, 0, *ok[10:]) == INVALID                            # 8 bits without scales
    assert f(*ok[:11], 100, 0) == TOO_SMALL


def test_quantise_and_weight_gradient_arguments():
    L = vb.lib()
    assert L.varco_quantize_rows(4, 60, 1, A, 64, A, 64, A, 3, 0) == INVALID
    assert L.varco_quantize_rows(4, 60, 1, A, 60, A, 64, A, 4, 0) == INVALID
    assert L.varco_quantize_rows(0, 60, 1, 0, 64, 0, 64, 0, 0, 0) == OK
    assert L.varco_quantize_weight(4, 60, 0, A, 59, A, 64, 0, 0, A, 1, 0) == INVALID
    assert L.varco_quantize_weight(4, 60, 0, A, 60, 0, 64, 0, 0, A, 1, 0) == INVALID
    assert L.varco_quantize_weight(4, 200, 0, A, 200, A, 208, 0, 0, A, 1, 0) == INVALID
    assert L.varco_weight_grad(4, 8, 8, 1, A, 8, A, 8, 0, 0, A, 1 << 40, 0) == INVALID
    assert L.varco_weight_grad(4, 8, 8, 1, A, 8, A, 8, A, 0, A, 512, 0) == TOO_SMALL
    assert L.varco_weight_grad(4, 8, 8, 1, A, 9, A, 8, A, 0, A, 1 << 40, 0) == INVALID
    assert L.varco_weight_grad(1 << 31, 8, 8, 1, A, 8, A, 8, A, 0, A, 1 << 40, 0) == UNSUPPORTED


def test_quantisers_refuse_what_their_grids_cannot_hold():
    """Widths whose count of blocks passes 65,535, up to the largest number, where rounding up to a block overflows 32 bits."""
    L = vb.lib()
    top, ld = (1 << 31) - 1, 1 << 31
    for F in (65535 * 128 + 1, top - 127, top - 126, top):
        assert L.varco_quantize_rows(4, F, 1, A, ld, A, ld, A, 4, 0) == UNSUPPORTED, F
        assert L.varco_quantize_weight(F, 4, 0, A, 4, A, 16, 0, 0, A, 1, 0) == UNSUPPORTED, F
    assert L.varco_quantize_weight(4, top, 0, A, top, A, ld, 0, 0, A, (1 << 24) - 1, 0) == INVALID       # too few scales a row
    assert L.varco_quantize_weight(4, top, 0, A, top, A, ld, 0, 0, A, 1 << 24, 0) == UNSUPPORTED


def test_clip_arguments():
    L = vb.lib()
    big = 1 << 22

    def arrays(g, n, t):
        k = len(g)
        return (C.c_void_p * k)(*g), (C.c_int64 * k)(*n), (C.c_int32 * k)(*t)
    g, n, t = arrays([A, A + 4], [10, 10], [0, 0])
    w = (C.c_void_p * 2)(A, A)
    assert L.varco_grad_norm(g, n, t, 2, 0, A, big, 0) == INVALID           # nowhere to put it
    assert L.varco_grad_norm(g, n, t, -1, A, A, big, 0) == INVALID
    assert L.varco_grad_norm(None, n, t, 2, A, A, big, 0) == INVALID
    assert L.varco_grad_norm(g, n, t, 2, A, A, 1000, 0) == TOO_SMALL
    assert L.varco_grad_norm(g, n, t, 1 << 20, A, A, big, 0) == UNSUPPORTED
    assert L.varco_grad_clip(g, n, t, 2, -1.0, 1e-6, 0, A, big, 0) == INVALID
    assert L.varco_grad_clip(g, n, t, 2, float("nan"), 1e-6, 0, A, big, 0) == INVALID
    assert L.varco_grad_clip(g, n, t, 2, 1.0, 0.0, 0, A, big, 0) == INVALID
    assert L.varco_clip_step(g, n, t, None, None, 2, 0.1, 1.0, 1e-6, 0, A, big, 0) == INVALID
    assert L.varco_clip_step(g, n, t, w, None, 2, float("nan"), 1.0, 1e-6, 0, A, big, 0) == INVALID
    for bad in (arrays([A, A + 2], [10, 10], [0, 0]), arrays([A, A + 1], [10, 10], [1, 1]), arrays([A, 0], [10, 10], [0, 0]),
                arrays([A, A], [10, -1], [0, 0]), arrays([A, A], [10, 10], [0, 3])):
        assert L.varco_grad_norm(*bad, 2, A, A, big, 0) == INVALID
    assert L.varco_clip_step(g, n, t, (C.c_void_p * 2)(A, A + 2), None, 2, 0.1, 1.0, 1e-6, 0, A, big, 0) == INVALID
    assert L.varco_clip_step(g, n, t, w, (C.c_void_p * 2)(A, A + 1), 2, 0.1, 1.0, 1e-6, 0, A, big, 0) == INVALID
