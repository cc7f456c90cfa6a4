"""GPU tests of the vocabulary losses (through the binding) against fp64.

Tolerances, before any run.  The softmax is formed as 2^(c z - c m) with
c = log2(e) / T: the argument is one fused multiply-add off a rounded c m, so
its error is at most 2^-23 of (|c z| + |c m|) and the value's relative error
ln 2 times that plus 2^-22 for the exponential; a sum of V such values adds at
most one 2^-24 for each addition on the longest path.  `rel` below bounds the
relative error of a probability by that sum.  Stored gradients add half a step
of their type (finfo.eps / 2).
The cross entropy's inputs are multiples of 1/2 and 1/4, so that every logit
is exact in fp32 and the bounds above are all there is: gradients in 16 bits are
sums of values rounded once to 16 bits (half a step each), in fp32.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -23


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("GPU tests need an MI355X; none is visible")
    import paper_2506_05960_amd as P
    P.load_library()
    yield


def losses(vocab, features=None, dtype="bf16", n=1):
    import paper_2506_05960_amd as P
    return P.VocabLoss(vocab, features=features, dtype=dtype, max_tokens=n)


def half_step(t, dt):
    f = torch.finfo(DT[dt])
    return t.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def within(got, want, bound):
    got, want = got.double().cpu(), want.cpu()
    return bool(((got - want).abs() <= bound.cpu()).all())


# ---- distillation ----

def distill64(z, ids, t, T, dloss):
    """loss, gradient, student and teacher probabilities (the latter over the vocabulary), from the definitions."""
    z, t = z.double().cpu(), t.double().cpu()
    ids, dloss = ids.cpu(), dloss.double().cpu()
    log_q = torch.log_softmax(z / T, dim=1)
    loss, P = torch.zeros(z.shape[0], dtype=torch.float64), torch.zeros_like(z)
    for r in range(z.shape[0]):
        use = (ids[r] >= 0) & (t[r] != -math.inf)
        if not bool(use.any()):
            continue
        lp = torch.log_softmax(t[r][use] / T, dim=0)
        at = ids[r][use].long()
        loss[r] = T * T * (lp.exp() * (lp - log_q[r, at])).sum()
        P[r].index_add_(0, at, lp.exp())
    live = (P.sum(dim=1) > 0).double()[:, None]
    grad = (dloss * T)[:, None] * (log_q.exp() - P) * live
    return loss, grad, log_q.exp(), P


def check_distill(z, ids, t, T, dloss, dtype, got_loss, got_grad):
    loss, grad, q, P = distill64(z, ids, t, T, dloss)
    V = z.shape[1]
    zf = z.double().cpu()
    c = math.log2(math.e) / T
    most = zf.masked_fill(zf.isinf(), 0).abs().amax(dim=1)
    tf = t.double().cpu()
    mt = tf.masked_fill(tf.isinf(), 0).abs().amax(dim=1)
    rel = U * (2 * c * torch.maximum(most, mt) + 4 + V / 256 + 24)[:, None]      # the longest run of additions
    g = (dloss.double().cpu() * T)[:, None].abs()
    gb = g * (q + P) * 2 * rel
    assert within(got_grad, grad, gb + half_step(grad.abs() + gb, dtype))
    size = 2 * c * (most + mt) + math.log2(V) + 8                                # |log2 p| + |log2 q| and their parts
    assert within(got_loss, loss, T * T * (2 * rel[:, 0] + 8 * U * size))


DISTILL = [  # n, vocab, top
    (1, 1, 1), (2, 5, 3), (3, 64, 64), (4, 513, 7), (7, 1000, 50), (5, 4099, 100), (2, 50021, 128), (3, 32768, 1),
    (300, 777, 20), (1, 160001, 16), (6, 2048, 1024),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,vocab,top", DISTILL)
def test_distill(n, vocab, top, dtype):
    g = torch.Generator().manual_seed(vocab + top)
    z = (torch.randn(n, vocab, generator=g) * 3).to(DT[dtype])
    ids = torch.stack([torch.randperm(vocab, generator=g)[:top] if top <= vocab else
                       torch.randint(0, vocab, (top,), generator=g) for _ in range(n)]).int()
    ids[torch.rand(n, top, generator=g) < 0.1] = -1
    t = (torch.randn(n, top, generator=g) * 2).to(DT[dtype])
    dloss = torch.rand(n, generator=g) + 0.5
    for T in (1.0, 2.5):
        loss, grad = losses(vocab, dtype=dtype, n=n).distill(z.cuda(), ids.cuda(), t.cuda(), T, dloss=dloss.cuda(),
                                                            grad=True)
        check_distill(z, ids, t, T, dloss, dtype, loss, grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_masks_and_duplicates(dtype):
    """Rows: nothing listed; nothing with a finite teacher logit; a token listed three times; a vocabulary masked to
    a few tokens by -infinity and by the type's lowest value; a teacher entry of -infinity."""
    V, lowest = 1003, torch.finfo(DT[dtype]).min
    g = torch.Generator().manual_seed(8)
    z = torch.randn(6, V, generator=g).to(DT[dtype])
    ids = torch.tensor([[-1, -1, -1, -1], [4, 5, 6, 7], [9, 1002, 9, 9], [0, 1, 2, 3], [0, 1, 2, 3], [500, 501, 3, -1]],
                       dtype=torch.int32)
    t = torch.randn(6, 4, generator=g).to(DT[dtype])
    t[1] = -math.inf
    z[3, 4:] = -math.inf
    z[4, 4:] = lowest
    t[5, 0] = -math.inf
    dloss = torch.ones(6)
    loss, grad = losses(V, dtype=dtype, n=6).distill(z.cuda(), ids.cuda(), t.cuda(), dloss=None, grad=True)
    assert float(loss[0]) == 0 and float(loss[1]) == 0 and bool((grad[:2] == 0).all())
    assert bool((grad[3:5, 4:] == 0).all())
    rows = torch.tensor([0, 1, 2, 3, 5])
    check_distill(z[rows], ids[rows], t[rows], 1.0, dloss[rows], dtype, loss[rows], grad[rows])
    # the lowest value behaves as a mask: its row equals the same row masked by infinities
    z[4, 4:] = -math.inf
    check_distill(z[4:5], ids[4:5], t[4:5], 1.0, dloss[:1], dtype, loss[4:5], grad[4:5])


def test_distill_refused_tokens_and_bad_rows_show():
    V = 300
    z, t = torch.randn(3, V, device="cuda"), torch.randn(3, 2, device="cuda")
    z[1, 7] = float("nan")
    ids = torch.tensor([[5, 6], [5, 6], [5, V]], dtype=torch.int32, device="cuda")
    loss, grad = losses(V, dtype="f32", n=3).distill(z, ids, t, grad=True)
    assert bool(loss[0].isfinite()) and bool(grad[0].isfinite().all())
    assert bool(loss[1:].isnan().all()) and bool(grad[1:].isnan().all())
    # a token that the student rules out and the teacher does not: infinite loss, its own gradient finite
    z = torch.zeros(1, V, device="cuda")
    z[0, 5] = -math.inf
    loss, grad = losses(V, dtype="f32", n=1).distill(z, ids[:1], t[:1], grad=True)
    assert float(loss) == math.inf and bool(grad.isfinite().all())


@pytest.mark.parametrize("n,vocab", [(3, 999), (2, 70001), (300, 2051)])
def test_distill_in_place_and_without_gradient(n, vocab):
    z = torch.randn(n, vocab, device="cuda").half()
    ids = torch.randint(0, vocab, (n, 9), device="cuda").int()
    t = torch.randn(n, 9, device="cuda").half()
    L = losses(vocab, dtype="f16", n=n)
    loss, grad = L.distill(z, ids, t, 1.5, grad=True)
    alone, none = L.distill(z, ids, t, 1.5)
    assert none is None and torch.equal(alone, loss)
    work = z.clone()
    again, same = L.distill(work, ids, t, 1.5, grad=work)
    assert same is work and torch.equal(again, loss) and torch.equal(work, grad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_distill_few_long_rows(dtype):
    """Rows that several workgroups share, at every offset from 16 bytes: listed tokens at both ends and at the ends of
    16-byte groups all along, some twice; rows masked but for a few tokens at the front, in the middle, at the back;
    a row without list; the gradient in place, alone and in graph replays."""
    V, top, n = 70003, 520, 11
    g = torch.Generator().manual_seed(21)
    z = (torch.randn(n, V, generator=g) * 2).to(DT[dtype])
    ids = torch.randint(0, V, (n, top), generator=g).int()
    ends = torch.arange(0, V, 137)[:500].int()
    ids[:, :500] = ends
    ids[:, 500:505] = torch.tensor([V - 1, V - 2, V - 9, 0, 1], dtype=torch.int32)
    t = torch.randn(n, top, generator=g).to(DT[dtype])
    live = {1: range(0, 3), 2: range(35000, 35004), 3: range(V - 3, V), 4: [5, 40000, V - 1]}
    for row, keep in live.items():
        keep = list(keep)
        z[row] = z[row].masked_fill(torch.ones(V, dtype=torch.bool).index_fill(0, torch.tensor(keep), False), -math.inf)
        ids[row] = -1
        ids[row, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
    ids[5] = -1
    dloss = torch.rand(n, generator=g) + 0.5
    L = losses(V, dtype=dtype, n=300)
    zg, ig, tg, dg = z.cuda(), ids.cuda(), t.cuda(), dloss.cuda()
    loss, grad = L.distill(zg, ig, tg, 1.5, dloss=dg, grad=True)
    check_distill(z, ids, t, 1.5, dloss, dtype, loss, grad)
    assert float(loss[5]) == 0 and bool((grad[5] == 0).all())
    for row, keep in live.items():
        assert int((grad[row] != 0).sum()) <= len(keep)
    work = zg.clone()
    again, _ = L.distill(work, ig, tg, 1.5, dloss=dg, grad=work)
    assert torch.equal(again, loss) and torch.equal(work, grad)
    assert torch.equal(L.distill(zg, ig, tg, 1.5, dloss=dg)[0], loss)
    out, dz = torch.empty_like(loss), torch.empty_like(grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.distill(zg, ig, tg, 1.5, dloss=dg, loss=out, grad=dz)
    for _ in range(3):
        L.distill(zg[:3], ig[:3], tg[:3], 1.0)                    # the workspace of another size in between
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, loss) and torch.equal(dz, grad)
        out.zero_()
        dz.zero_()


@pytest.mark.parametrize("n", [1, 17, 64, 65, 255, 256, 257])
def test_distill_row_counts(n):
    """A row's loss does not depend on how many rows there are, beyond the order of its sums."""
    V, top = 33003, 7
    g = torch.Generator().manual_seed(n)
    z = torch.randn(1, V, generator=g).to(torch.bfloat16)
    ids = torch.randint(0, V, (1, top), generator=g).int()
    t = torch.randn(1, top, generator=g).to(torch.bfloat16)
    loss, grad = losses(V, n=n).distill(z.repeat(n, 1).cuda(), ids.repeat(n, 1).cuda(), t.repeat(n, 1).cuda(), grad=True)
    check_distill(z, ids, t, 1.0, torch.ones(1), "bf16", loss[-1:], grad[-1:])
    assert bool((loss - loss[0]).abs().max() <= 2e-5) and bool((grad.float() - grad[0].float()).abs().max() <= 2.0 ** -8)


def test_distill_bad_rows_show_in_segments():
    V = 40001
    z, t = torch.randn(4, V, device="cuda"), torch.randn(4, 2, device="cuda")
    z[1, 39000] = float("nan")
    z[3, 100] = float("inf")
    ids = torch.tensor([[5, 6], [5, 6], [5, V], [7, 8]], dtype=torch.int32, device="cuda")
    loss, grad = losses(V, dtype="f32", n=4).distill(z, ids, t, grad=True)
    assert bool(loss[0].isfinite()) and bool(grad[0].isfinite().all())
    assert bool(loss[1:3].isnan().all()) and bool(grad[1:3].isnan().all()) and not bool(loss[3].isfinite())


def test_distill_gradient_matches_differences():
    """Central differences of the loss in fp32: their own error is the third-order term, |step|^2 / 6 of a smooth
    function whose third derivatives are at most 1, plus the losses' rounding over the step."""
    V, step = 40, 2.0 ** -5
    g = torch.Generator().manual_seed(3)
    z = torch.randn(1, V, generator=g)
    ids = torch.tensor([[3, 17, 3, 39, -1]], dtype=torch.int32, device="cuda")
    t = torch.randn(1, 5, generator=g).cuda()
    L = losses(V, dtype="f32", n=2 * V)
    _, grad = L.distill(z.cuda(), ids, t, 2.0, grad=True)
    moved = z.repeat(2 * V, 1)
    moved[torch.arange(V), torch.arange(V)] += step
    moved[torch.arange(V) + V, torch.arange(V)] -= step
    loss, _ = L.distill(moved.cuda(), ids.repeat(2 * V, 1), t.repeat(2 * V, 1), 2.0)
    slope = (loss[:V] - loss[V:]).double() / (2 * step)
    assert float((slope - grad[0].double()).abs().max()) <= step * step / 6 + 64 * U * float(loss.max()) / step


# ---- cross entropy ----

def ce_inputs(n, F, V, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-2, 3, (n, F), generator=g).float() / 2
    w = torch.randint(-2, 3, (V, F), generator=g).float() / 4
    if F > 64:                                   # logits of a few units
        x[:, 64:] *= (torch.rand(n, F - 64, generator=g) < 0.1).float()
    targets = torch.randint(0, V, (n,), generator=g)
    targets[torch.rand(n, generator=g) < 0.15] = -100
    dloss = torch.rand(n, generator=g) + 0.5
    return x.to(DT[dtype]).cuda(), w.to(DT[dtype]).cuda(), targets.cuda(), dloss.cuda()


def check_ce(x, w, targets, dloss, dtype, loss, dx, dw):
    n, V = x.shape[0], w.shape[0]
    x, w, dl = x.double(), w.double(), dloss.double()
    z = x @ w.t()
    counts = targets >= 0
    log_p = torch.log_softmax(z, dim=1)
    rows = torch.arange(n, device="cuda")[counts]
    want = torch.zeros(n, dtype=torch.float64, device="cuda")
    want[rows] = -log_p[rows, targets[counts]]
    most = z.abs().amax(dim=1)
    rel = U * (2 * 1.4427 * most + 4 + V / 256 + 300)[:, None]     # 256 values a tile, then the tiles, then lanes
    assert within(loss, want, counts * (2 * rel[:, 0] + 8 * U * (4 * most + math.log2(V + 1) + 8)))
    p = log_p.exp()
    dz = p.clone()
    dz[rows, targets[counts]] -= 1
    weight = (dl * counts)[:, None]
    # one rounding of dz (a fp16 dz after the scaling that takes the largest weight past 2^14) and p's own error
    tiny = 2.0 ** -25 * float(dl.abs().max()) * 2.0 ** -14 if dtype == "f16" else 2.0 ** -134
    dz, ddz = dz * weight, weight * (dz.abs() * (torch.finfo(DT[dtype]).eps / 2) + 2 * (p + (dz - p).abs()) * rel) + tiny
    if dx is not None:
        want, b = dz @ w, ddz @ w.abs() + (V + 64) * U * (dz.abs() @ w.abs())
        assert within(dx, want, b + half_step(want.abs() + b, dtype))
        assert bool((dx[~counts] == 0).all())
    if dw is not None:
        want, b = dz.t() @ x, ddz.t() @ x.abs() + (n + 64) * U * (dz.t().abs() @ x.abs())
        assert within(dw, want, b + half_step(want.abs() + b, dtype))


CE = [  # n, features, vocab
    (1, 8, 1), (1, 8, 2), (3, 16, 255), (5, 64, 256), (64, 72, 257), (100, 576, 999), (255, 136, 1300), (257, 64, 4097),
    (300, 264, 700), (2, 64, 20011),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,F,V", CE)
def test_cross_entropy(n, F, V, dtype):
    x, w, targets, dloss = ce_inputs(n, F, V, dtype, n + V)
    L = losses(V, F, dtype, n)
    loss, dx, dw = L.cross_entropy(x, w, targets, dloss, dx=True, dw=True)
    check_ce(x, w, targets, dloss, dtype, loss, dx, dw)
    again = L.cross_entropy(x, w, targets, dloss, dx=True, dw=True)
    assert all(torch.equal(a, b) for a, b in zip(again, (loss, dx, dw)))
    alone, none, none_ = L.cross_entropy(x, w, targets, dloss)
    assert none is None and none_ is None and torch.equal(alone, loss)
    for got in (L.cross_entropy(x, w, targets, dloss, dx=True), L.cross_entropy(x, w, targets, dloss, dw=True)):
        check_ce(x, w, targets, dloss, dtype, *got)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_cross_entropy_in_pieces(dtype):
    """max_tokens of 2^18 leaves 256 vocabulary rows a piece."""
    n, F, V = 130, 72, 1100
    x, w, targets, dloss = ce_inputs(n, F, V, dtype, 9)
    L = losses(V, F, dtype, 1 << 18)
    check_ce(x, w, targets, dloss, dtype, *L.cross_entropy(x, w, targets, dloss, dx=True, dw=True))
    check_ce(x, w, targets, dloss, dtype, *L.cross_entropy(x, w, targets, dloss, dx=True))


@pytest.mark.parametrize("scale", [1e-6, 3e4])
def test_cross_entropy_weights_of_any_size(scale):
    """fp16 gradients keep their relative precision through small and large row weights."""
    n, F, V = 40, 64, 600
    x, w, targets, dloss = ce_inputs(n, F, V, "bf16", 5)
    xh, wh = x.half(), w.half()
    dloss = dloss * scale
    _, dx, dw = losses(V, F, "bf16", n).cross_entropy(x, w, targets, dloss, dx=True, dw=True)
    check_ce(x, w, targets, dloss, "bf16", losses(V, F, "bf16", n).cross_entropy(x, w, targets, dloss)[0], dx, dw)
    if scale < 1:
        got = losses(V, F, "f16", n).cross_entropy(xh, wh, targets, dloss, dx=True, dw=True)
        check_ce(xh, wh, targets, dloss, "f16", *got)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("units", [1, 2, 3, 5, 8])
def test_cross_entropy_stores_the_largest_target_entry_exactly(units, dtype):
    """Two tokens, dz = +-q with q = dloss / (1 + e^gap): the stored entries are exact, and the gradients are off by
    their own rounding, q's (`rel`: exponentials, sums and the difference from 1, 2^-23 over q) and the fp32 products'."""
    F = 64
    x, w = torch.zeros(1, F), torch.zeros(2, F)
    x[0, :units], x[0, units:] = 0.5, 0
    w[0, :units], w[1, :units] = 0.5, 0.25
    w[:, units:] = torch.randint(-4, 5, (2, F - units), generator=torch.Generator().manual_seed(units)) / 4
    dl = torch.tensor([0.7])
    L = losses(2, features=F, dtype=dtype, n=1)
    _, dx, dw = L.cross_entropy(x.to(DT[dtype]).cuda(), w.to(DT[dtype]).cuda(), torch.tensor([0], device="cuda"),
                                dloss=dl.cuda(), dx=True, dw=True)
    q = float(dl.double()) / (1 + math.exp(units / 8))
    dz = torch.tensor([[-q, q]], dtype=torch.float64)
    for got, want in ((dx, dz @ w.double()), (dw, dz.t() @ x.double())):
        assert within(got, want, half_step(want, dtype) + want.abs() * (64 * U * (1 + 0.7 / q)))


def test_cross_entropy_rows_that_do_not_count():
    n, F, V = 70, 64, 300
    x, w, targets, dloss = ce_inputs(n, F, V, "bf16", 2)
    L = losses(V, F, "bf16", n)
    want = L.cross_entropy(x, w, targets, dloss, dx=True, dw=True)
    # whatever an uncounted position holds stays there
    x[targets < 0] = float("nan")
    got = L.cross_entropy(x, w, targets, dloss, dx=True, dw=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    none = torch.full_like(targets, -1)
    loss, dx, dw = L.cross_entropy(x, w, none, dloss, dx=True, dw=True)
    assert bool((loss == 0).all()) and bool((dx == 0).all()) and bool((dw == 0).all())
    # a target past the vocabulary shows
    x, w, targets, dloss = ce_inputs(n, F, V, "bf16", 2)
    targets[3], targets[4] = V, 0
    loss, dx, _ = L.cross_entropy(x, w, targets, None, dx=True)
    assert bool(loss[3].isnan()) and bool(dx[3].isnan().all()) and bool(loss[4].isfinite())
    assert bool(dx[torch.arange(n, device="cuda") != 3].isfinite().all())


def test_cross_entropy_extreme_logits():
    """Logits of some hundreds: the loss is their difference, the probabilities zeros and ones."""
    n, F, V = 4, 8, 520
    x = torch.zeros(n, F, device="cuda").bfloat16()
    w = torch.zeros(V, F, device="cuda").bfloat16()
    x[:, 0] = 16
    w[7, 0], w[500, 0], w[:, 1] = 32, -32, 1
    targets = torch.tensor([7, 500, 0, -1], device="cuda")
    loss, dx, _ = losses(V, F, "bf16", n).cross_entropy(x, w, targets, dx=True)
    assert loss.tolist() == [0.0, 1024.0, 512.0, 0.0]
    assert bool((dx[0] == 0).all()) and float(dx[1, 0]) == 64 and float(dx[2, 0]) == 32


def test_cross_entropy_gradient_matches_differences():
    n, F, V, step = 1, 8, 30, 2.0 ** -4
    x, w, _, _ = ce_inputs(1, F, V, "f16", 1)
    targets = torch.tensor([11], device="cuda")
    L = losses(V, F, "f16", 2 * F)
    _, dx, _ = L.cross_entropy(x, w, targets, dx=True)
    moved = x.repeat(2 * F, 1)
    moved[torch.arange(F), torch.arange(F)] += step
    moved[torch.arange(F) + F, torch.arange(F)] -= step
    loss, _, _ = L.cross_entropy(moved, w, targets.repeat(2 * F))
    slope = (loss[:F] - loss[F:]).double() / (2 * step)
    # third derivatives of the loss along x_i are at most max|w|^3, and dX is rounded to fp16 after sums of rounded values
    third = float(w.abs().max()) ** 3
    bound = step * step / 6 * third + 64 * U * float(loss.max()) / step + 2.0 ** -11 * 3 * float(w.abs().max())
    assert float((slope - dx[0].double()).abs().max()) <= bound


def test_first_gradient_under_capture_is_refused():
    import paper_2506_05960_amd as P
    n, F, V = 9, 16, 40
    x, w, targets, dloss = ce_inputs(n, F, V, "bf16", 3)
    L = losses(V, F, "bf16", n)
    loss, dx = torch.empty(n, device="cuda"), torch.empty_like(x)
    want, _, _ = L.cross_entropy(x, w, targets, dloss)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(P.AQError, match="capture"):
            L.cross_entropy(x, w, targets, dloss, loss=loss, dx=dx)
        L.cross_entropy(x, w, targets, dloss, loss=loss)      # the loss alone needs nothing more
    loss.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, want)


@pytest.mark.parametrize("n", [1, 40, 65, 130, 257, 700])
def test_token_counts_below_the_most(n):
    """Handles made for many tokens serve fewer: their plans differ, their workspace holds each."""
    F, V = 136, 3000
    x, w, targets, dloss = ce_inputs(n, F, V, "f16", n)
    L = losses(V, F, "f16", 700)
    check_ce(x, w, targets, dloss, "f16", *L.cross_entropy(x, w, targets, dloss, dx=True, dw=True))


def test_losses_on_another_stream_and_in_graphs():
    n, F, V = 90, 72, 1031
    L = losses(V, F, "bf16", n)
    sets = [ce_inputs(n, F, V, "bf16", s) for s in range(3)]
    lists = [(torch.randn(n, V, device="cuda").bfloat16(), torch.randint(-1, V, (n, 11), device="cuda").int(),
              torch.randn(n, 11, device="cuda").bfloat16()) for _ in range(3)]
    want = [[t.clone() for t in L.cross_entropy(*s, dx=True, dw=True)] + list(L.distill(*m, 2.0, grad=True))
            for s, m in zip(sets, lists)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = list(L.cross_entropy(*sets[1], dx=True, dw=True)) + list(L.distill(*lists[1], 2.0, grad=True))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
    ins = [t.clone() for t in sets[0] + lists[0]]
    outs = [torch.empty_like(t) for t in want[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.cross_entropy(*ins[:4], loss=outs[0], dx=outs[1], dw=outs[2])
        L.distill(*ins[4:], 2.0, loss=outs[3], grad=outs[4])
    for r in range(6):
        for t, s in zip(ins, sets[r % 3] + lists[r % 3]):
            t.copy_(s)
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want[r % 3]))
