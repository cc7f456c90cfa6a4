"""GPU tests of the vocabulary losses at the ends of their ranges, against fp64."""
import math

import pytest
import torch

import test_gpu_losses as TL

pytestmark = pytest.mark.gpu

DT = TL.DT


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("GPU tests need an MI355X; none is visible")
    import paper_2506_05960_amd as P
    P.load_library()
    yield


@pytest.mark.parametrize("T", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("vocab", [1003, 70001])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_distill_lists_a_token_masked_by_the_lowest_value(dtype, vocab, T):
    """The teacher lists a token that the student's mask sets to its type's lowest value: the loss is p times that
    value and some units, T (p is below a quarter: within fp32).

    Bound, relative: the loss is p |lowest| T but for terms an eighth of it (fp16) or less, of the same p and of
    logarithms good to some 2^-20; p's relative error is 2^-23 of the exponents' size (2 log2(e) / T 4 units: 23) and of its sum's (4 + 24); differences,
    products and the sum add 2^-23 each, 60 in all; 2^-17."""
    n, lowest = 5, torch.finfo(DT[dtype]).min
    g = torch.Generator().manual_seed(vocab)
    z = torch.randn(n, vocab, generator=g).clamp(-4, 4).to(DT[dtype])
    ids = torch.tensor([[7, 900, 3, 5, 11]], dtype=torch.int32).repeat(n, 1)
    t = torch.tensor([[-2.0, 1.0, 0.5, 0.25, 0.0]]).repeat(n, 1).to(DT[dtype])
    z[:, 7] = lowest
    z[2:, 20:500] = lowest
    loss, grad = TL.losses(vocab, dtype=dtype, n=n).distill(z.cuda(), ids.cuda(), t.cuda(), T, grad=True)
    want, want_grad, q, P = TL.distill64(z, ids, t, T, torch.ones(n))
    assert bool(want.float().isfinite().all()) and bool((P[:, 7] < 0.25).all())
    assert TL.within(loss, want, want.abs() * 2.0 ** -17)
    b = T * (q + P) * 2.0 ** -16
    assert TL.within(grad, want_grad, b + TL.half_step(want_grad.abs() + b, dtype))
