"""GPU tests of the 4-bit layers and the vocabulary losses at sizes that take
every kernel variant: large tiles of the dense product, wide and long layers of
few tokens, many and long rows of the distillation.  Which sizes take which
variant is held by the launches' shapes in ``test_usq_losses_routes_host.py``.

The bounds are those of ``test_gpu_usq.py`` and ``test_gpu_losses.py``.
"""
import pytest
import torch

import test_gpu_losses as TL
import test_gpu_usq as TU
from test_usq_losses_routes_host import CE_ROUTES, DISTILL_ROUTES, FEW_ROUTES, GRAD_ROUTES

pytestmark = pytest.mark.gpu

DT = TU.DT


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("GPU tests need an MI355X; none is visible")
    import paper_2506_05960_amd as P
    P.load_library()
    yield


# ---- 4-bit layers ----

@pytest.mark.parametrize("dtype,y,group", [("f16", "f32", 32), ("bf16", "bf16", 64), ("bf16", "f32", 128)])
@pytest.mark.parametrize("K,C_out", sorted({(K, C_out) for _, K, C_out, _, _ in FEW_ROUTES}))
def test_few_tokens(K, C_out, group, dtype, y):
    """On both sides of every change of the rows a workgroup takes, the last workgroup's row tiles repeated or not."""
    codes, scales, z, W, mag = TU.make(K, C_out, group, dtype, True, seed=K + C_out)
    lay = TU.layer_of(codes, scales, z, group, dtype, y, 64)
    g = torch.Generator().manual_seed(C_out)
    Wg, mg = W.t().cuda(), mag.t().cuda()
    for n in (1, 4, 5, 16, 17, 32, 33, 64):
        x = torch.randn(n, K, generator=g).to(DT[dtype])
        out = torch.full((n + 1, C_out), 7.0, dtype=DT[y], device="cuda")
        got = lay.forward(x.cuda(), out=out[:n]).double()
        want = x.double().cuda() @ Wg
        bound = (2 * K + 8) * TU.U32 * (x.double().abs().cuda() @ mg)
        bound = bound + TU.half_step(want.abs() + bound, y)
        assert bool(((got - want).abs() <= bound).all()), n
        assert bool((out[n] == 7).all())


@pytest.mark.parametrize("dtype,group", [("f16", 32), ("bf16", 64), ("f16", 128), ("bf16", 256)])
@pytest.mark.parametrize("n,K,C_out", [(1100, 392, 300), (2100, 264, 130), (70, 4104, 520)])
def test_many_tokens(n, K, C_out, group, dtype):
    """More than eight tiles of tokens (two bands of them), and K in several splits."""
    codes, scales, z, W, mag = TU.make(K, C_out, group, dtype, True, seed=n)
    lay = TU.layer_of(codes, scales, z, group, dtype, "f32", n)
    x = torch.randn(n, K, generator=torch.Generator().manual_seed(n)).to(DT[dtype]).cuda()
    out = torch.full((n + 1, C_out), 7.0, device="cuda")
    got = lay.forward(x, out=out[:n]).double()
    want = x.double() @ W.t().cuda()
    bound = (2 * K + 8) * TU.U32 * (x.double().abs() @ mag.t().cuda())
    assert bool(((got - want).abs() <= bound + TU.half_step(want.abs() + bound, "f32")).all())
    assert bool((out[n] == 7).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,K,C_out", [r[:3] for r in GRAD_ROUTES])
def test_input_grad(n, K, C_out, dtype):
    codes, scales, z, W, _ = TU.make(K, C_out, 64, dtype, True, seed=n)
    lay = TU.layer_of(codes, scales, z, 64, dtype, dtype, n)
    dy = torch.randn(n, C_out, generator=torch.Generator().manual_seed(n)).to(DT[dtype])
    out = torch.full((n + 1, K), 7.0, dtype=DT[dtype], device="cuda")
    got = lay.input_grad(dy.cuda(), out=out[:n]).double()
    W, d = W.cuda(), dy.double().cuda()
    want = d @ W
    bound = d.abs() @ TU.half_step(W, dtype) + (C_out + 8) * TU.U32 * (d.abs() @ W.abs())
    assert bool(((got - want).abs() <= bound + TU.half_step(want.abs() + bound, dtype)).all())
    assert bool((out[n] == 7).all())


# ---- cross entropy ----

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,F,V,most", [r[:4] for r in CE_ROUTES])
def test_cross_entropy(n, F, V, most, dtype):
    x, w, targets, dloss = TL.ce_inputs(n, F, V, dtype, n + V)
    targets[:4] = torch.tensor([0, V - 1, V - 1, 255])
    L = TL.losses(V, F, dtype, most)
    loss, dx, dw = L.cross_entropy(x, w, targets, dloss, dx=True, dw=True)
    TL.check_ce(x, w, targets, dloss, dtype, loss, dx, dw)
    again = L.cross_entropy(x, w, targets, dloss, dx=True, dw=True)
    assert all(torch.equal(a, b) for a, b in zip(again, (loss, dx, dw)))
    for got in (L.cross_entropy(x, w, targets, dloss, dx=True), L.cross_entropy(x, w, targets, dloss, dw=True)):
        TL.check_ce(x, w, targets, dloss, dtype, *got)


# ---- distillation ----

@pytest.mark.parametrize("n,vocab,dtype", sorted({r[:3] for r in DISTILL_ROUTES if r[0] > 1}))
def test_distill(n, vocab, dtype):
    top = 9
    g = torch.Generator().manual_seed(vocab + n)
    z = (torch.randn(n, vocab, generator=g) * 2).to(DT[dtype])
    ids = torch.randint(0, vocab, (n, top), generator=g).int()
    ids[:, 0], ids[:, 1] = 0, vocab - 1
    ids[3] = -1
    t = torch.randn(n, top, generator=g).to(DT[dtype])
    dloss = torch.rand(n, generator=g) + 0.5
    L = TL.losses(vocab, dtype=dtype, n=n)
    zg, ig, tg, dg = z.cuda(), ids.cuda(), t.cuda(), dloss.cuda()
    loss, grad = L.distill(zg, ig, tg, 1.5, dloss=dg, grad=True)
    rows = torch.cat([torch.arange(0, n, 37), torch.tensor([3, n - 1])])
    TL.check_distill(z[rows], ids[rows], t[rows], 1.5, dloss[rows], dtype, loss[rows], grad[rows])
    # every row, as one number: softmax and the teacher's mass both sum to one, but for half a step of each stored value
    # (at least half the smallest) and the probabilities' own errors, less than 2^-16 at logits below 12
    f = torch.finfo(DT[dtype])
    size = grad.double().abs().sum(dim=1)
    lim = (f.eps / 2 + 2.0 ** -16) * size + vocab * f.smallest_normal * f.eps / 2
    assert bool((z.abs() < 12).all()) and bool((grad.double().sum(dim=1).abs() <= lim).all())
    assert torch.equal(L.distill(zg, ig, tg, 1.5, dloss=dg)[0], loss)
    again, _ = L.distill(zg, ig, tg, 1.5, dloss=dg, grad=zg)
    assert torch.equal(again, loss) and torch.equal(zg, grad)


def test_many_tokens_offsets_past_32_bits():
    """Outputs of 2.2 thousand million values: 128 tokens over and over, so that every block repeats the first."""
    n, wide = 128 * 1100, 16000
    assert n * wide > 1 << 31
    for K, C_out, call in ((8, wide, "forward"), (wide, 8, "input_grad")):
        codes, scales, z, W, mag = TU.make(K, C_out, 128, "bf16", True, seed=9)
        lay = TU.layer_of(codes, scales, z, 128, "bf16", "bf16", n)
        x = torch.randn(128, 8, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        got = getattr(lay, call)(x.repeat(n // 128, 1))
        W64 = W.t().cuda() if call == "forward" else W.cuda()
        want = x.double() @ W64
        bound = 24 * TU.U32 * (x.double().abs() @ (mag.t().cuda() if call == "forward" else W64.abs()))
        if call == "input_grad":
            bound = bound + x.double().abs() @ TU.half_step(W64, "bf16")
        assert bool(((got[:128].double() - want).abs() <= bound + TU.half_step(want.abs() + bound, "bf16")).all())
        for at in [*range(128, n, 128 * 97), n - 128]:
            assert torch.equal(got[at:at + 128], got[:128])
        lay.close()
        del got
