"""Overlaps and workspaces of the 4-bit layers and the vocabulary losses, on the host path alone (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import host_device
from paper_2506_05960_amd import aq as A

I = A.AQ_ERR_INVALID_ARGUMENT


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    A.load_library()
    return host_device.build(tmp_path_factory)


def distill_overlaps(vocab, dtype, n):
    """Statuses of calls whose loss lies at, before, behind and clear of dloss."""
    lib, h, P = A.load_library(), ctypes.c_void_p(), 1 << 20
    assert lib.aq_loss_create(ctypes.byref(A.aq_loss_desc(vocab, 0, dtype, n)), ctypes.byref(h)) == A.AQ_OK
    got = [lib.aq_loss_distill(h, 4096, 4096, 4096, 2, 1.0, P, P + off, 4096, n, None)
           for off in (0, 4 * (n - 1), -4 * (n - 1), 4 * n, -4 * n)]
    lib.aq_loss_destroy(h)
    return got


@pytest.mark.parametrize("vocab, dtype, n, at", [
    (40001, A.AQ_F32, 4, I), (70003, A.AQ_BF16, 100, I), (131072, A.AQ_F16, 2, I),       # segments: several workgroups a row
    (300, A.AQ_F32, 4, 0), (50000, A.AQ_BF16, 600, 0)])                                 # one, which reads dloss first
def test_distillation_refuses_a_loss_over_dloss(so, vocab, dtype, n, at):
    got = host_device.in_child(so, "test_usq_losses_workspace_host", "distill_overlaps", vocab, dtype, n)
    assert got == [at, I, I, 0, 0]


def usq_gradient_bytes(K, C_out, most):
    """Bytes held after a layer's input gradients of 1, `most` and 17 tokens, and the splits (the second
    dimension of the last launch of one workgroup column a chunk) of `most` tokens."""
    lib, h = A.load_library(), ctypes.c_void_p()
    d = A.aq_usq_desc(C_out, K, 128, A.AQ_F16, A.AQ_F16, most)
    codes, scales = np.zeros((C_out, K // 2), np.uint8), np.zeros((C_out, -(-K // 128)), np.uint16)
    assert lib.aq_usq_create(ctypes.byref(d), codes.ctypes.data, scales.ctypes.data, None, ctypes.byref(h)) == A.AQ_OK
    live, got, splits = host_device.live_bytes(), [], 0
    for n in (1, most, min(most, 17)):
        st, launched = host_device.launches(lambda: lib.aq_usq_input_grad(h, 4096, 4096, n, None))
        assert st == A.AQ_OK
        got.append(host_device.live_bytes() - live)
        if n == most:
            splits = [y for x, y, *_ in launched if x == -(-K // 128)][-1]
    lib.aq_usq_destroy(h)
    return got, splits


@pytest.mark.parametrize("K, C_out, most, slab", [
    (4096, 16384, 64, False), (576, 1155, 64, False), (4096, 16384, 1, False), (1 << 20, 16, 1, False),
    (576, 1155, 65, True), (4096, 4096, 4096, True), (1 << 20, 16, 64, True)])
def test_layers_of_few_tokens_hold_no_decoded_weights(so, K, C_out, most, slab):
    """Fp32 sums of each split and, for uneven rows, dY's copy; a slab is all of these layers' weights in 16 bits."""
    got, splits = host_device.in_child(so, "test_usq_losses_workspace_host", "usq_gradient_bytes", K, C_out, most)
    assert got[0] == got[1] == got[2]
    padded = -(-C_out // 8) * 8
    copy = 2 * most * padded if C_out % 8 else 0
    if slab:
        assert got[0] >= 2 * K * padded + copy
    else:
        assert got[0] == 4 * most * K * splits + copy


def temperatures(values):
    lib, h = A.load_library(), ctypes.c_void_p()
    assert lib.aq_loss_create(ctypes.byref(A.aq_loss_desc(300, 0, A.AQ_F32, 4)), ctypes.byref(h)) == A.AQ_OK
    got = [lib.aq_loss_distill(h, 4096, 4096, 4096, 2, t, None, 4096, 4096, 4, None) for t in values]
    lib.aq_loss_destroy(h)
    return got


def test_temperatures_without_a_finite_reciprocal_are_refused(so):
    """log2(e) / T scales the logits: an infinity makes NaN of every row's largest logit."""
    got = host_device.in_child(so, "test_usq_losses_workspace_host", "temperatures", [2.0 ** -149, 2.0 ** -128, 2.0 ** -127, 1e30])
    assert got == [A.AQ_ERR_UNSUPPORTED, A.AQ_ERR_UNSUPPORTED, A.AQ_OK, A.AQ_OK]


def test_descriptors_refuse_what_would_wrap_from_below_or_in_64_bits():
    codes, scales = np.zeros((24, 32), np.uint8), np.ones((24, 2), np.float16)
    with pytest.raises(ValueError, match="vocab is past -2\\^31"):
        A.VocabLoss(5 - (1 << 32), max_tokens=2)
    for most in ((1 << 64) + 4, 4 - (1 << 64)):
        with pytest.raises(ValueError, match="max_tokens is past -?2\\^63"):
            A.VocabLoss(5, max_tokens=most)
        with pytest.raises(ValueError, match="max_tokens is past -?2\\^63"):
            A.USQLayer(codes, scales, group=32, max_tokens=most)
