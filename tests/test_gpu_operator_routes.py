"""GPU tests of the 4-bit layers at sizes that take every kernel variant: wide and
long layers of few tokens.  Which sizes take which variant is held by the
launches' shapes in ``test_usq_losses_routes_host.py``.

The bounds are those of ``test_gpu_usq.py``.
"""
import pytest
import torch

import test_gpu_usq as TU
from test_usq_losses_routes_host import FEW_ROUTES

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
