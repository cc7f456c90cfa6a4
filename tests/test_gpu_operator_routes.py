"""GPU tests of the 4-bit layers and the distillation at sizes that take every
kernel variant: wide and long layers of few tokens, many and long rows.  Which
sizes take which variant is held by the launches' shapes in
``test_usq_losses_routes_host.py``.

The bounds are those of ``test_gpu_usq.py`` and ``test_gpu_losses.py``.
"""
import pytest
import torch

import test_gpu_losses as TL
import test_gpu_usq as TU
from test_usq_losses_routes_host import DISTILL_ROUTES, FEW_ROUTES

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
