"""GPU tests of the 4-bit layers (through the binding) against fp64.

Forward: codes minus zero points are small integers, products of them with
the 16-bit inputs are exact in fp32, so an output differs from the exact one
by its fp32 sums (at most one unit of 2^-23 relative to the sum of magnitudes
for each of the K products, of the group sums that carry the zero points and of
the scalings) and by its own rounding (half a step, finfo.eps / 2).
Input gradient: the weights are rounded once to the layer's type besides.
A one-hot input selects one weight, which has to come out exactly.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
U32 = 2.0 ** -23


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("GPU tests need an MI355X; none is visible")
    import paper_2506_05960_amd as P
    P.load_library()
    yield


def make(K, C_out, group, dtype, zeros, seed=0):
    """(codes, scales, zeros, W in fp64 [C_out, K], magnitudes s * (q + z))."""
    g = torch.Generator().manual_seed(seed)
    G = -(-K // group)
    q = torch.randint(0, 16, (C_out, K), generator=g, dtype=torch.uint8)
    scales = ((torch.rand(C_out, G, generator=g) + 0.5) / 8).to(DT[dtype])
    z = torch.randint(0, 16, (C_out, G), generator=g, dtype=torch.uint8) if zeros else None
    j = torch.arange(K) // group
    z64 = z.double()[:, j] if zeros else torch.full((C_out, K), 8.0, dtype=torch.float64)
    s64 = scales.double()[:, j]
    return q[:, 0::2] | (q[:, 1::2] << 4), scales, z, s64 * (q.double() - z64), s64 * (q.double() + z64)


def layer_of(codes, scales, z, group, dtype, y, n):
    import paper_2506_05960_amd as P
    return P.USQLayer(codes, scales, z, group=group, dtype=dtype, y_dtype=y, max_tokens=n)


def half_step(t, dt):
    """Half a step of type ``dt`` at each value, its smallest subnormal step included."""
    f = torch.finfo(DT[dt])
    return t.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


SHAPES = [  # n, K, C_out, group
    (1, 8, 1, 32), (1, 128, 16, 128), (1, 4096, 130, 128), (2, 1000, 33, 128), (5, 264, 17, 32), (16, 576, 48, 64),
    (17, 520, 31, 64), (33, 2304, 65, 256), (64, 640, 129, 128), (65, 136, 250, 32), (130, 384, 257, 128),
    (257, 904, 300, 64), (520, 1024, 513, 256), (300, 8, 700, 64),
]


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype,y", [("f16", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("n,K,C_out,group", SHAPES)
def test_forward(n, K, C_out, group, dtype, y, zeros):
    codes, scales, z, W, mag = make(K, C_out, group, dtype, zeros, seed=K + C_out)
    lay = layer_of(codes, scales, z, group, dtype, y, n)
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, K, generator=g).to(DT[dtype])
    got = lay.forward(x.cuda())
    assert got.dtype == DT[y] and got.shape == (n, C_out)
    want = x.double() @ W.t()
    bound = (2 * K + 8) * U32 * (x.double().abs() @ mag.t())
    bound = bound + half_step(want.abs() + bound, y)
    assert bool(((got.cpu().double() - want).abs() <= bound).all())
    assert torch.equal(lay.forward(x.cuda()), got)          # fixed order of sums
    lay.close()


@pytest.mark.parametrize("n,K,C_out,group,dtype", [(1, 264, 40, 32, "f16"), (40, 264, 40, 64, "bf16"),
                                                  (256, 1152, 264, 128, "bf16"), (200, 520, 70, 32, "f16")])
def test_one_hot_inputs_select_exact_weights(n, K, C_out, group, dtype):
    codes, scales, z, W, _ = make(K, C_out, group, dtype, True, seed=3)
    lay = layer_of(codes, scales, z, group, dtype, "f32", n)
    at = torch.randperm(K, generator=torch.Generator().manual_seed(4))[:n]
    at = torch.cat([at, torch.arange(n - at.numel()) % K])
    x = torch.zeros(n, K, dtype=DT[dtype])
    x[torch.arange(n), at] = 1
    assert torch.equal(lay.forward(x.cuda()).cpu().double(), W[:, at].t())


@pytest.mark.parametrize("n", [1, 20, 80, 300])
def test_special_inputs_stay_in_their_rows(n):
    """An infinity or a NaN in one token's input reaches that token's outputs alone."""
    K, C_out = 392, 70
    codes, scales, z, W, _ = make(K, C_out, 128, "bf16", True)
    lay = layer_of(codes, scales, z, 128, "bf16", "f32", n)
    x = torch.randn(n, K, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    clean = lay.forward(x.cuda()).cpu()
    x[n // 2, K - 1] = float("nan")
    got = lay.forward(x.cuda()).cpu()
    assert bool(got[n // 2].isnan().all())
    keep = torch.arange(n) != n // 2
    assert torch.equal(got[keep], clean[keep])


def test_rows_behind_the_output_stay():
    """A forward over fewer tokens than the buffer holds leaves the others' rows as they were."""
    K, C_out = 256, 37
    codes, scales, z, _, _ = make(K, C_out, 64, "f16", False)
    lay = layer_of(codes, scales, z, 64, "f16", "f16", 400)
    for n in (1, 7, 70, 300):
        buf = torch.full((400, C_out), 7.0, dtype=torch.float16, device="cuda")
        lay.forward(torch.randn(n, K, device="cuda").half(), out=buf[:n])
        assert bool((buf[n:] == 7).all())
        gbuf = torch.full((400, K), 7.0, dtype=torch.float16, device="cuda")
        lay.input_grad(torch.randn(n, C_out, device="cuda").half(), out=gbuf[:n])
        assert bool((gbuf[n:] == 7).all())


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,K,C_out,group", [(1, 8, 1, 32), (3, 136, 8, 32), (33, 264, 77, 64), (200, 520, 130, 128),
                                             (257, 904, 264, 256), (300, 1152, 576, 64), (600, 384, 1000, 128),
                                             (1, 1000, 1031, 64), (15, 264, 2000, 32), (16, 128, 128, 128), (17, 136, 129, 64),
                                             (32, 640, 4100, 256), (49, 72, 31, 32), (64, 2312, 515, 64), (64, 520, 16, 384),
                                             (65, 520, 515, 64)])
def test_input_grad(n, K, C_out, group, dtype, zeros):
    codes, scales, z, W, _ = make(K, C_out, group, dtype, zeros, seed=K * C_out)
    lay = layer_of(codes, scales, z, group, dtype, dtype, n)
    dy = torch.randn(n, C_out, generator=torch.Generator().manual_seed(n)).to(DT[dtype])
    got = lay.input_grad(dy.cuda())
    want = dy.double() @ W
    bound = dy.double().abs() @ half_step(W, dtype) + (C_out + 8) * U32 * (dy.double().abs() @ W.abs())
    bound = bound + half_step(want.abs() + bound, dtype)
    assert got.dtype == DT[dtype] and got.shape == (n, K)
    assert bool(((got.cpu().double() - want).abs() <= bound).all())
    assert torch.equal(lay.input_grad(dy.cuda()), got)


@pytest.mark.parametrize("n, K, C_out", [(40, 1304, 40000), (5, 600, 125000), (70, 1304, 40000), (70, 600, 125000)])
def test_input_grad_in_slabs(n, K, C_out):
    """Layers whose decoded weights come near the workspace's 128 MiB, and pass them."""
    codes, scales, z, W, _ = make(K, C_out, 128, "bf16", True)
    lay = layer_of(codes, scales, z, 128, "bf16", "bf16", n)
    dy = torch.randn(n, C_out, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    got = lay.input_grad(dy.cuda()).cpu().double()
    Wd, d = W.cuda(), dy.double().cuda()
    want = (d @ Wd).cpu()
    bound = (d.abs() @ half_step(Wd, "bf16") + (C_out + 8) * U32 * (d.abs() @ Wd.abs())).cpu()
    assert bool(((got - want).abs() <= bound + half_step(want.abs() + bound, "bf16")).all())


def test_input_grad_matches_differences_of_the_forward():
    """dX . e is the change of sum(dY * Y) along e; integer-valued inputs keep every sum exact."""
    n, K, C_out = 9, 256, 64
    g = torch.Generator().manual_seed(5)
    q = torch.randint(4, 13, (C_out, K), generator=g, dtype=torch.uint8)
    codes, scales = q[:, 0::2] | (q[:, 1::2] << 4), torch.full((C_out, 4), 0.125, dtype=torch.float16)
    lay = layer_of(codes, scales, None, 64, "f16", "f32", n)
    x = torch.randint(-2, 3, (n, K), generator=g).half().cuda()
    e = torch.randint(-1, 2, (n, K), generator=g).half().cuda()
    dy = torch.randint(-1, 2, (n, C_out), generator=g).half().cuda()
    slope = ((lay.forward(x + e) - lay.forward(x)).double() * dy.double()).sum()
    dx = lay.input_grad(dy)
    assert float((dx.double() * e.double()).sum()) == float(slope)


@pytest.mark.parametrize("n", [37, 90])
def test_another_stream_and_graph_replays(n):
    K, C_out = 520, 131
    codes, scales, z, _, _ = make(K, C_out, 64, "bf16", True)
    lay = layer_of(codes, scales, z, 64, "bf16", "bf16", n)
    xs = [torch.randn(n, K, device="cuda").bfloat16() for _ in range(3)]
    ds = [torch.randn(n, C_out, device="cuda").bfloat16() for _ in range(3)]
    want = [(lay.forward(x), lay.input_grad(d)) for x, d in zip(xs, ds)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = lay.forward(xs[0])
    side.synchronize()
    assert torch.equal(y, want[0][0])
    x, d = xs[0].clone(), ds[0].clone()
    y, dx = torch.empty_like(want[0][0]), torch.empty_like(want[0][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lay.forward(x, out=y)
        lay.input_grad(d, out=dx)
    for r in range(6):
        x.copy_(xs[r % 3])
        d.copy_(ds[r % 3])
        y.zero_()
        dx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[r % 3][0]) and torch.equal(dx, want[r % 3][1])


def test_first_gradient_under_capture_is_refused():
    import paper_2506_05960_amd as P
    codes, scales, z, _, _ = make(128, 24, 32, "f16", False)
    lay = layer_of(codes, scales, z, 32, "f16", "f16", 4)
    dy, dx, t = torch.ones(4, 24, device="cuda").half(), torch.empty(4, 128, device="cuda").half(), torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(P.AQError, match="capture"):
            lay.input_grad(dy, out=dx)
        t += 1
    graph.replay()
    torch.cuda.synchronize()
    assert float(t.sum()) == 4
    lay.input_grad(dy, out=dx)               # outside: allocates and runs


def test_numpy_arrays_and_raw_bf16_bits():
    codes, scales, z, _, _ = make(128, 24, 32, "bf16", True)
    x = torch.randn(3, 128, device="cuda").bfloat16()
    a = layer_of(codes, scales, z, 32, "bf16", "f32", 3).forward(x)
    b = layer_of(codes.numpy(), scales.view(torch.int16).numpy().view(np.uint16), z.numpy(), 32, "bf16", "f32", 3).forward(x)
    assert torch.equal(a, b)
