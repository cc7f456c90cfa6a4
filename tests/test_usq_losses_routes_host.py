"""Which kernels calls of the 4-bit layers and the vocabulary losses take, by their launches' shapes (no GPU needed).

The GPU tests of these routes (``test_gpu_operator_routes.py``) take their sizes from here, so that a change of the
plans that leaves a variant without a test shows."""
import ctypes

import numpy as np
import pytest

import host_device
from paper_2506_05960_amd import aq as A

BIG, SMALL = 512, 256        # threads of the dense product's 256 x 256 and 128 x 128 tiles

# few tokens: n, K, C_out, output rows a workgroup takes (16 a row tile), waves
FEW_ROUTES = [
    (1, 264, 4096, 16, 3), (4, 264, 12288, 16, 3), (1, 264, 12305, 32, 3), (1, 4104, 4096, 16, 8), (4, 4104, 4101, 32, 8),
    (5, 264, 12288, 16, 3), (16, 264, 12305, 32, 3), (16, 4104, 4096, 16, 8), (5, 4104, 4101, 32, 8),
    (17, 264, 4096, 16, 3), (32, 264, 4101, 32, 3), (17, 264, 8192, 32, 3), (32, 264, 8209, 64, 3),
    (33, 264, 4096, 16, 3), (64, 264, 4101, 32, 3), (33, 264, 8192, 32, 3), (64, 264, 8209, 64, 3),
    (3, 8200, 300, 16, 16), (9, 8200, 300, 16, 16), (1, 8200, 4101, 32, 8), (16, 8200, 4101, 32, 8), (64, 8200, 300, 16, 8),
]

# input gradients: n, K, C_out, threads of the product's workgroups, its workgroups
GRAD_ROUTES = [(2100, 4104, 4099, BIG, 9 * 17), (513, 4104, 8195, BIG, 5 * 3 * 17), (300, 4104, 4099, SMALL, 5 * 3 * 33),
               (1100, 2312, 4099, SMALL, 9 * 19)]

# cross entropy: n, features, vocab, max_tokens; threads of the statistics, and of the gradient, dX and dW products of
# each piece; K splits of dX; pieces
CE_ROUTES = [
    (1030, 136, 9001, 1030, BIG, BIG, SMALL, SMALL, 13, 1),
    (2100, 4104, 2100, 2100, SMALL, SMALL, BIG, BIG, 1, 1),
    (130, 4104, 9001, 130, SMALL, SMALL, BIG, BIG, 15, 1),
    (2100, 4104, 1100, 1 << 17, SMALL, SMALL, BIG, SMALL, 1, 3),
    (130, 72, 1100, 1 << 18, SMALL, SMALL, SMALL, SMALL, 1, 5),
    (5, 64, 5001, 1 << 15, SMALL, SMALL, SMALL, SMALL, 28, 3),
]

# distillation: n, vocab, dtype, launches, threads of the last one
DISTILL_ROUTES = [
    (1, 32767, "f32", 1, 512), (1, 32768, "f32", 2, 256), (128, 32768, "bf16", 2, 256), (129, 32768, "bf16", 1, 512),
    (129, 98303, "f16", 1, 512), (129, 98304, "f16", 2, 256), (192, 98309, "bf16", 2, 256), (193, 98309, "bf16", 1, 512),
    (512, 2003, "bf16", 1, 512), (513, 2003, "f32", 1, 256), (513, 2003, "f16", 1, 256), (513, 40003, "bf16", 1, 256),
    (514, 57351, "f16", 1, 256), (513, 57353, "bf16", 1, 512), (513, 16387, "f32", 1, 256), (513, 17001, "f32", 1, 512),
    (257, 60001, "f16", 1, 512), (257, 60003, "bf16", 1, 512), (257, 30001, "f32", 1, 512),
]


def _usq(n, K, C_out, group=128, call="aq_usq_forward"):
    """Grid and block of each launch of a layer's second call over n tokens."""
    lib, h = A.load_library(), ctypes.c_void_p()
    d = A.aq_usq_desc(C_out, K, group, A.AQ_BF16, A.AQ_BF16, n)
    codes, scales = np.zeros((C_out, K // 2), np.uint8), np.zeros((C_out, -(-K // group)), np.uint16)
    assert lib.aq_usq_create(ctypes.byref(d), codes.ctypes.data, scales.ctypes.data, None, ctypes.byref(h)) == A.AQ_OK
    f = getattr(lib, call)
    assert f(h, 4096, 4096, n, None) == A.AQ_OK
    st, out = host_device.launches(lambda: f(h, 4096, 4096, n, None))
    assert st == A.AQ_OK
    lib.aq_usq_destroy(h)
    return [(x, y, b) for x, y, _, b, *_ in out]


def few(routes, group):
    return [_usq(n, K, C_out, group) for n, K, C_out, *_ in routes]


def grads(routes):
    return [_usq(n, K, C_out, 64, "aq_usq_input_grad") for n, K, C_out, *_ in routes]


def cross_entropies(routes):
    lib, out = A.load_library(), []
    for n, F, V, most, *_ in routes:
        h = ctypes.c_void_p()
        assert lib.aq_loss_create(ctypes.byref(A.aq_loss_desc(V, F, A.AQ_BF16, most)), ctypes.byref(h)) == A.AQ_OK
        st, got = host_device.launches(lambda: lib.aq_loss_cross_entropy(h, 4096, 4096, 4096, None, 4096, 4096, 4096, n, None))
        assert st == A.AQ_OK
        lib.aq_loss_destroy(h)
        out.append([(x, b) for x, _, _, b, *_ in got])
    return out


def distills(routes):
    lib, out = A.load_library(), []
    for n, V, dtype, *_ in routes:
        h = ctypes.c_void_p()
        assert lib.aq_loss_create(ctypes.byref(A.aq_loss_desc(V, 0, A.DTYPE_CODES[dtype], n)), ctypes.byref(h)) == A.AQ_OK
        st, got = host_device.launches(lambda: lib.aq_loss_distill(h, 4096, 4096, 4096, 9, 1.0, None, 4096, 4096, n, None))
        assert st == A.AQ_OK
        lib.aq_loss_destroy(h)
        out.append([len(got), got[-1][3]])
    return out


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    A.load_library()
    return host_device.build(tmp_path_factory)


@pytest.mark.parametrize("group", [64, 128])
def test_few_token_routes(so, group):
    for route, got in zip(FEW_ROUTES, host_device.in_child(so, "test_usq_losses_routes_host", "few", FEW_ROUTES, group)):
        n, K, C_out, rows, waves = route
        if n > 32 and group < 128:
            rows = min(rows, 32)
        assert got == [[-(-C_out // rows), 1, 64 * waves]], route


def test_distillation_routes(so):
    got = host_device.in_child(so, "test_usq_losses_routes_host", "distills", DISTILL_ROUTES)
    assert got == [[launches, threads] for *_, launches, threads in DISTILL_ROUTES]


def test_input_gradient_routes(so):
    for route, got in zip(GRAD_ROUTES, host_device.in_child(so, "test_usq_losses_routes_host", "grads", GRAD_ROUTES)):
        n, K, C_out, threads, wgs = route
        assert [wgs, 1, threads] in got, (route, got)


def test_cross_entropy_routes(so):
    for route, got in zip(CE_ROUTES, host_device.in_child(so, "test_usq_losses_routes_host", "cross_entropies", CE_ROUTES)):
        n, F, V, most, stats, grad, dx, dw, splits, pieces = route
        tiles = lambda M, N, threads: -(-M // (128 if threads == SMALL else 256)) * -(-N // (128 if threads == SMALL else 256))
        assert got[0] == [tiles(V, n, stats), stats]
        per = got[2:]
        join = 1 if splits > 1 else 0
        assert len(per) == 3 * pieces + join, (route, got)
        at = 0
        for p in range(pieces):
            g, x = per[at], per[at + 1]
            assert g[1] == grad and x[1] == dx and x[0] == tiles(n, F, dx) * splits, (route, got)
            at += 2 + (join if p + 1 == pieces else 0)
            assert per[at][1] == dw, (route, got)
            at += 1
