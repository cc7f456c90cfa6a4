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
