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


@pytest.mark.parametrize("both", [True, False])
@pytest.mark.parametrize("n,V", [(40, 30011), (200, 2003)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_cross_entropy_rows_of_far_smaller_weights(dtype, n, V, both):
    """Weights from 2^12 down to 2^-12 in one call: each row of dX against its own bound.

    A row's stored dz is rounded once: half a step, at least half the smallest subnormal step (2^-25 in fp16) under the
    scale that takes the row's entry at its target to 32640 (just below 2^15: 2^-39 of that entry).  p and the sums as in
    test_gpu_losses.py.  The head's weights are positive, so that errors of one sign add up."""
    F = 64
    x, w, targets, _ = TL.ce_inputs(n, F, V, dtype, 31)
    w = w.abs()
    dloss = 2.0 ** torch.linspace(12, -12, n).round().cuda()
    L = TL.losses(V, F, dtype, n)
    loss, dx, dw = L.cross_entropy(x, w, targets, dloss, dx=True, dw=both)
    TL.check_ce(x, w, targets, dloss, dtype, loss, None, dw)
    x, w, counts = x.double(), w.double(), targets >= 0
    z = x @ w.t()
    p = torch.softmax(z, dim=1)
    dz = p.clone()
    rows = torch.arange(n, device="cuda")[counts]
    dz[rows, targets[counts]] -= 1
    weight = (dloss.double() * counts)[:, None]
    rel = TL.U * (2 * 1.4427 * z.abs().amax(dim=1) + 4 + V / 256 + 300)[:, None]
    peak = torch.zeros(n, 1, dtype=torch.float64, device="cuda")
    peak[rows, 0] = dz[rows, targets[counts]].abs().clamp(min=2.0 ** -20)        # (less is rounding)
    eps = torch.finfo(DT[dtype]).eps
    ddz = weight * (dz.abs() * (eps / 2) + 2 * (p + (dz - p).abs()) * rel + peak * 2.0 ** -39)
    want, b = (weight * dz) @ w, ddz @ w + (V + 64) * TL.U * ((weight * dz).abs() @ w)
    assert TL.within(dx, want, b + TL.half_step(want.abs() + b, dtype))


def test_distill_offsets_past_32_bits():
    """2.2 thousand million logits: 64 rows over and over, so that every block of 64 has to repeat the first."""
    V, n, top = 131073, 64 * 263, 5
    assert n * V > 1 << 31
    g = torch.Generator().manual_seed(3)
    z = torch.randn(64, V, generator=g).to(torch.bfloat16)
    ids = torch.randint(0, V, (64, top), generator=g).int()
    ids[:, 0] = V - 1
    t = torch.randn(64, top, generator=g).to(torch.bfloat16)
    many = z.cuda().repeat(n // 64, 1)
    loss, grad = TL.losses(V, n=n).distill(many, ids.cuda().repeat(n // 64, 1), t.cuda().repeat(n // 64, 1), 1.5, grad=many)
    rows = torch.tensor([0, 31, 63])
    TL.check_distill(z[rows], ids[rows], t[rows], 1.5, torch.ones(3), "bf16", loss[rows], grad[rows])
    assert torch.equal(loss, loss[:64].repeat(n // 64))
    for at in range(64, n, 64 * 37):
        assert torch.equal(grad[at:at + 64], grad[:64])
    assert torch.equal(grad[-64:], grad[:64])


def test_cross_entropy_offsets_past_32_bits():
    """A head of 4.5 GB: 1000 rows over and over, the targets in the last ones.  Bounds as in test_gpu_losses.py."""
    n, F, unique, times = 5, 4096, 1000, 550
    V = unique * times
    assert V * F * 2 > 1 << 32
    x, w, _, dloss = TL.ce_inputs(n, F, unique, "bf16", 12)
    targets = torch.tensor([V - 1, V - 1000, 0, V - 500, -1], device="cuda")
    loss, dx, dw = TL.losses(V, F, "bf16", n).cross_entropy(x, w.repeat(times, 1), targets, dloss, dx=True, dw=True)
    z, counts = x.double() @ w.double().t(), targets >= 0
    log_p = torch.log_softmax(z, dim=1) - math.log(times)
    at = targets.clamp(min=0) % unique
    rows = torch.arange(n, device="cuda")
    most = z.abs().amax(dim=1)
    rel = TL.U * (2 * 1.4427 * most + 4 + V / 256 + 300)
    assert TL.within(loss, -log_p[rows, at] * counts, counts * (2 * rel + 8 * TL.U * (4 * most + math.log2(V) + 8)))
    # the tokens' own rows of dz, over the unique rows (for dX their sum over the repeats) and at the targets
    weight = (dloss.double() * counts)[:, None]
    p = log_p.exp()
    one = torch.zeros_like(p)
    one[rows, at] = 1
    half = torch.finfo(torch.bfloat16).eps / 2
    want = (weight * (p * times - one)) @ w.double()
    size = (weight * (p * times + one)) @ w.double().abs()
    assert TL.within(dx, want, size * (half + 2 * float(rel.max()) + (V + 64) * TL.U) + TL.half_step(want, "bf16"))
    for first in (0, unique * (times // 2), V - unique):
        here = one * ((targets >= first) & (targets < first + unique))[:, None]
        want = (weight * (p - here)).t() @ x.double()
        size = (weight * (p + here)).t() @ x.double().abs()
        got = dw[first:first + unique]
        assert TL.within(got, want, size * (half + 2 * float(rel.max()) + 128 * TL.U) + TL.half_step(want.abs() + size * half, "bf16"))
