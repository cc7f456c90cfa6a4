"""A tuning step of a low-bit model, end to end on the library's own calls:
an additively quantized layer, a head (4-bit, or dense and unquantised), a loss
over the vocabulary, and the gradients back to the layer's codebooks, against
the same chain in fp64.

Every intermediate is stored in fp16 (eps / 2 = 2^-11 of its value): the layer's
output, the head's logits, the logits' gradient, the head's input gradient, and
the head's rounded weights.  Errors of logits of a few units move probabilities
by that much again, so the bar for the codebook gradient is an infinity-norm
relative error of 2 * (5 roundings + 4 units of logits) * 2^-11 = 9e-3.
"""
import numpy as np
import pytest
import torch

import oracle as O
from workloads import LayerSpec, generate

pytestmark = pytest.mark.gpu

TOL = 9e-3
N, K, HIDDEN, VOCAB = 96, 256, 192, 1003


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("GPU tests need an MI355X; none is visible")
    import paper_2506_05960_amd as P
    P.load_library()
    yield


def _body(seed):
    import paper_2506_05960_amd as P
    spec = LayerSpec(name="tuned", C_out=HIDDEN, K=K, g=8, M=2, B=8, n=N, codebook_std=0.04)
    inp = generate(spec, seed)
    x = torch.from_numpy(np.ascontiguousarray(inp["x"])).cuda()
    return P.AQLayer(spec, inp), spec, inp, x


def _codebook_grad64(spec, inp, x, dh):
    """dC of the layer for the output gradient ``dh`` (fp64), by the definition."""
    dW = (dh.t() @ x.double()) * torch.from_numpy(inp["scales"]).double().cuda()[:, None]
    codes = torch.from_numpy(inp["codes"].astype(np.int64)).cuda()
    dC = torch.zeros(spec.M, 1 << spec.B, spec.g, dtype=torch.float64, device="cuda")
    for m in range(spec.M):
        dC[m].index_add_(0, codes[:, :, m].reshape(-1), dW.reshape(-1, spec.g))
    return dC


def _hidden64(spec, inp, x):
    return torch.from_numpy(O.forward(spec, inp)).double().cuda()


def _close(got, want):
    err = float((got.double() - want).abs().max() / want.abs().max())
    print(f"  codebook gradient rel_inf {err:.2e}", flush=True)
    assert err <= TOL


def test_distilling_through_a_4bit_head():
    import paper_2506_05960_amd as P
    body, spec, inp, x = _body(21)
    g = torch.Generator().manual_seed(4)
    q = torch.randint(0, 16, (VOCAB, HIDDEN), generator=g, dtype=torch.uint8)
    scales = ((torch.rand(VOCAB, 3, generator=g) + 0.5) / 64).half()
    zeros = torch.randint(6, 10, (VOCAB, 3), generator=g, dtype=torch.uint8)
    head = P.USQLayer(q[:, 0::2] | (q[:, 1::2] << 4), scales, zeros, group=64, dtype="f16", max_tokens=N)
    ids = torch.stack([torch.randperm(VOCAB, generator=g)[:12] for _ in range(N)]).int().cuda()
    teacher = torch.randn(N, 12, generator=g).half().cuda()
    L = P.VocabLoss(VOCAB, dtype="f16", max_tokens=N)

    h = body.forward(x)
    z = head.forward(h)
    loss, dz = L.distill(z, ids, teacher, 2.0, grad=True)
    dh = head.input_grad(dz)
    got = body.codebook_grad(x, dh)

    j = torch.arange(HIDDEN) // 64
    W = (scales.double()[:, j] * (q.double() - zeros.double()[:, j])).cuda()
    z64 = _hidden64(spec, inp, x) @ W.t()
    p = torch.zeros_like(z64).scatter_(1, ids.long(), torch.softmax(teacher.double() / 2, dim=1))
    dz64 = 2 * (torch.softmax(z64 / 2, dim=1) - p)
    _close(got, _codebook_grad64(spec, inp, x, dz64 @ W))


@pytest.mark.parametrize("captured", [False, True])
def test_cross_entropy_of_an_unquantised_head(captured):
    import paper_2506_05960_amd as P
    body, spec, inp, x = _body(22)
    g = torch.Generator().manual_seed(5)
    W = (torch.randn(VOCAB, HIDDEN, generator=g) / 8).half().cuda()
    targets = torch.randint(0, VOCAB, (N,), generator=g).cuda()
    targets[::7] = -1
    L = P.VocabLoss(VOCAB, features=HIDDEN, dtype="f16", max_tokens=N)
    h = torch.empty(N, HIDDEN, dtype=torch.float16, device="cuda")
    dh, dW, loss = torch.empty_like(h), torch.empty_like(W), torch.empty(N, device="cuda")
    dC = torch.empty(spec.M, 1 << spec.B, spec.g, device="cuda")

    def step():
        body.forward(x, out=h)
        L.cross_entropy(h, W, targets, loss=loss, dx=dh, dw=dW)
        body.codebook_grad(x, dh, out=dC)

    step()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(3):
            for t in (h, dh, dW, loss, dC):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
    z64 = _hidden64(spec, inp, x) @ W.double().t()
    dz = torch.softmax(z64, dim=1)
    rows = torch.arange(N, device="cuda")[targets >= 0]
    dz[rows, targets[rows]] -= 1
    dz[targets < 0] = 0
    _close(dC, _codebook_grad64(spec, inp, x, dz @ W.double()))
    want = dz.t() @ _hidden64(spec, inp, x)
    assert float((dW.double() - want).abs().max() / want.abs().max()) <= TOL
