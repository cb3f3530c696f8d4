"""Global gradient norm, clipping and the clipped step against 64 bits.  The norm's sixteen-term partial sums round in fp32
(16 u of them), everything after that in 64 bits, and the norm itself rounds once: 2^-20 covers it.  A step rounds the
factor (4 u) and one fused multiply-add."""
import pytest
import torch

from paper_2406_17611_b200 import binding as vb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


def tensors(sizes, dtype, seed, scale=1.0, offset=0):
    """Tensors of the sizes in one storage; with an offset, starting at odd elements."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    out, at = [], offset
    flat = (torch.randn(sum(sizes) + offset * (len(sizes) + 1) + 64, generator=g, device=DEV) * scale).to(dtype)
    for n in sizes:
        out.append(flat[at:at + n])
        at += n + offset
    return out


def norm64(ts):
    return float(sum((t.double() ** 2).sum() for t in ts).sqrt())


SIZES = {"one": [1], "few": [7, 1, 100, 0, 33], "layers": [25600, 25600, 256, 65536, 65536, 256, 12032, 12032, 47],
         "many": [(i * 37) % 301 + 1 for i in range(700)], "more than a table": [(i * 53) % 97 + 1 for i in range(1700)], "large": [3000001, 8, 5000000, 16385], "none": [0, 0]}


@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("name", list(SIZES))
def test_norm_clip_and_step(name, dtype, offset):
    sizes = SIZES[name]
    ws = vb.varco_ops_workspace()
    g = tensors(sizes, dtype, 5, 1e-2, offset)
    want = norm64(g)
    n = vb.varco_grad_norm(g, ws)
    assert abs(float(n) - want) <= 2.0 ** -20 * want
    for max_norm in (0.3 * want + 1e-9, 10 * want + 1.0):
        c = min(1.0, max_norm / (want + 1e-6))
        w = tensors(sizes, torch.float32, 6, 1.0, offset)
        cp = tensors(sizes, torch.bfloat16, 7, 1.0, offset)
        w64 = [x.double() for x in w]
        before = [x.clone() for x in g]
        m = vb.varco_clip_step(w, g, 0.5, max_norm, copies=[x if i % 3 else None for i, x in enumerate(cp)], workspace=ws)
        assert abs(float(m) - want) <= 2.0 ** -20 * want
        for i, (a, b, x) in enumerate(zip(w, w64, g)):
            k = 0.5 * c * x.double()
            assert bool(((a.double() - (b - k)).abs() <= 2 * U * b.abs() + 2.0 ** -19 * k.abs()).all())
            assert torch.equal(cp[i], a.bfloat16()) or i % 3 == 0
        assert all(torch.equal(x, y) for x, y in zip(g, before))
        h = [x.clone() for x in g]
        m = vb.varco_grad_clip(h, max_norm, ws)
        assert abs(float(m) - want) <= 2.0 ** -20 * want
        round_ = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -19
        for a, x in zip(h, g):
            if c == 1.0:
                assert torch.equal(a, x)
            else:
                assert bool(((a.double() - c * x.double()).abs() <= round_ * c * x.double().abs()).all())


def test_neighbouring_memory_is_left_alone():
    ws = vb.varco_ops_workspace()
    flat = torch.ones(4096, device=DEV)
    w = torch.ones(4096, device=DEV)
    vb.varco_clip_step([w[5:1000], w[1001:4000]], [flat[5:1000], flat[1001:4000]], 1.0, 1e9, workspace=ws)
    assert bool((w[:5] == 1).all()) and float(w[1000]) == 1 and bool((w[4000:] == 1).all()) and not w[5:1000].any() and not w[1001:4000].any()
    vb.varco_grad_clip([flat[5:1000]], 0.0, ws)
    assert bool((flat[:5] == 1).all()) and bool((flat[1000:] == 1).all()) and not flat[5:1000].any()


def test_norm_outside_the_range_of_squares():
    ws = vb.varco_ops_workspace()
    for v in (1e30, 1e-30, 3e38, 1e-37, 1e-44):
        t = torch.full((1000,), v, device=DEV)
        want = norm64([t])
        n = float(vb.varco_grad_norm([t], ws).double())
        assert n == float("inf") if want > 3.4e38 else abs(n - want) <= 2.0 ** -20 * want + 1e-45
    mix = [torch.full((33,), 1e25, device=DEV), torch.full((5000,), 1.0, device=DEV)]
    assert abs(float(vb.varco_grad_norm(mix, ws)) - norm64(mix)) <= 2.0 ** -20 * norm64(mix)


def test_not_finite_gradients():
    ws = vb.varco_ops_workspace()
    a, b = torch.ones(100, device=DEV), torch.ones(50, device=DEV)
    a[7] = float("inf")
    w = [torch.ones(100, device=DEV), torch.ones(50, device=DEV)]
    assert float(vb.varco_clip_step(w, [a, b], 0.1, 1.0, workspace=ws)) == float("inf")
    assert bool(torch.isnan(w[0][7])) and int(torch.isnan(w[0]).sum()) == 1 and bool((w[1] == 1).all())
    a[7] = float("nan")
    assert torch.isnan(vb.varco_grad_norm([a, b], ws)).item()
    vb.varco_grad_clip([b, a], 1.0, ws)
    assert bool(torch.isnan(b).all())


def test_reproducible():
    ws = vb.varco_ops_workspace()
    g = tensors([1234567, 99, 2000003], torch.float32, 8)
    assert torch.equal(vb.varco_grad_norm(g, ws), vb.varco_grad_norm(g, ws))


def test_a_barrier_that_the_others_never_reach_ends():
    """Counters that no number of arrivals completes: the wait runs out after its second, the status says so, weights and norm stay
    as they were, and the workspace works again once it is zeroed."""
    ws = vb.varco_ops_workspace()
    word = (-ws.data_ptr()) % 256 // 4 + 32               # of the aligned base: status at 0, barrier at 128 bytes
    w, g = torch.ones(100000, device=DEV), torch.ones(100000, device=DEV)
    ws[:1024].view(torch.int32)[word] = 1 << 30
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    vb.varco_clip_step([w], [g], 0.5, 1e9, workspace=ws)
    end.record()
    assert vb.varco_workspace_status(ws) == 31
    assert bool((w == 1).all()) and 500 < start.elapsed_time(end) < 5000
    ws.zero_()
    assert abs(float(vb.varco_clip_step([w], [g], 0.5, 1e9, workspace=ws)) - 100000 ** 0.5) <= 2.0 ** -20 * 100000 ** 0.5
    assert bool((w == 0.5).all()) and vb.varco_workspace_status(ws) == 0


def test_refusals():
    ws = vb.varco_ops_workspace()
    t, bad = torch.ones(64, device=DEV), pytest.raises((ValueError, TypeError, vb.VarcoError))
    with bad:
        vb.varco_grad_norm([t.half()], ws)
    with bad:
        vb.varco_grad_norm([t.cpu()], ws)
    with bad:
        vb.varco_grad_norm([t[::2]], ws)
    with bad:
        vb.varco_grad_norm([t, t], ws)
    with bad:
        vb.varco_grad_norm([t], ws[:100])
    with bad:
        vb.varco_grad_norm([t], None)
    with bad:
        vb.varco_grad_norm([], ws)
    with bad:
        vb.varco_grad_clip([t], -1.0, ws)
    with bad:
        vb.varco_grad_clip([t], 1.0, ws, eps=0.0)
    with bad:
        vb.varco_clip_step([t, t], [t], 1.0, 1.0, workspace=ws)
    with bad:
        vb.varco_clip_step([t[:32]], [t], 1.0, 1.0, workspace=ws)
    with bad:
        vb.varco_clip_step([t.bfloat16()], [t], 1.0, 1.0, workspace=ws)
    with bad:
        vb.varco_clip_step([t.clone()], [t], 1.0, 1.0, copies=[t.clone()], workspace=ws)
