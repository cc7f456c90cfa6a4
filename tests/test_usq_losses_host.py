"""Refusals of the 4-bit layers and the vocabulary losses, before anything is launched (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import host_device
from paper_2506_05960_amd import aq as A

C_OUT, K, VOCAB, F = 24, 64, 300, 64


def _lib():
    return A.load_library()


def _create_usq(no=None, zeros=None, **change):
    d = dict(out_features=C_OUT, in_features=K, group=32, dtype=A.AQ_F16, y_dtype=A.AQ_F16, max_tokens=8)
    d.update(change)
    buf = np.zeros(1 << 16, np.uint8)
    args = [ctypes.byref(A.aq_usq_desc(**d)), buf.ctypes.data, buf.ctypes.data,
            None if zeros is None else zeros.ctypes.data]
    if no is not None:
        args[no] = None
    h = ctypes.c_void_p(1234)
    st = _lib().aq_usq_create(*args, ctypes.byref(h))
    return st, h.value, _lib().aq_last_error().decode()


@pytest.mark.parametrize("change, status, text", [
    (dict(out_features=0), A.AQ_ERR_INVALID_ARGUMENT, "out_features"),
    (dict(in_features=0), A.AQ_ERR_INVALID_ARGUMENT, "in_features"),
    (dict(group=0), A.AQ_ERR_INVALID_ARGUMENT, "group"),
    (dict(dtype=9), A.AQ_ERR_INVALID_ARGUMENT, "dtype"),
    (dict(y_dtype=A.AQ_I8), A.AQ_ERR_INVALID_ARGUMENT, "y_dtype"),
    (dict(max_tokens=0), A.AQ_ERR_INVALID_ARGUMENT, "max_tokens"),
    (dict(dtype=A.AQ_F32), A.AQ_ERR_UNSUPPORTED, "fp16 or bf16"),
    (dict(in_features=60), A.AQ_ERR_UNSUPPORTED, "multiple of 8"),
    (dict(group=16), A.AQ_ERR_UNSUPPORTED, "group"),
    (dict(group=96), A.AQ_ERR_UNSUPPORTED, "group"),
    (dict(group=192), A.AQ_ERR_UNSUPPORTED, "group"),
    (dict(max_tokens=1 << 40), A.AQ_ERR_UNSUPPORTED, "2^24"),
    (dict(out_features=(1 << 21) + 1), A.AQ_ERR_UNSUPPORTED, "2^21"),
    (dict(in_features=(1 << 21) + 8), A.AQ_ERR_UNSUPPORTED, "2^21"),
])
def test_usq_create_refuses(change, status, text):
    st, h, msg = _create_usq(**change)
    assert st == status and text in msg and h is None


def test_usq_create_refuses_null_and_bad_zero_points():
    for i in range(3):
        st, h, msg = _create_usq(no=i)
        assert st == A.AQ_ERR_INVALID_ARGUMENT and "null" in msg and h is None
    zeros = np.full((C_OUT, 2), 15, np.uint8)
    zeros[-1, -1] = 16
    st, h, msg = _create_usq(zeros=zeros)
    assert st == A.AQ_ERR_INVALID_ARGUMENT and "zero point" in msg and h is None


def _create_loss(**change):
    d = dict(vocab=VOCAB, features=F, dtype=A.AQ_BF16, max_tokens=8)
    d.update(change)
    h = ctypes.c_void_p(1234)
    st = _lib().aq_loss_create(ctypes.byref(A.aq_loss_desc(**d)), ctypes.byref(h))
    return st, h.value, _lib().aq_last_error().decode()


@pytest.mark.parametrize("change, status, text", [
    (dict(vocab=0), A.AQ_ERR_INVALID_ARGUMENT, "vocab"),
    (dict(features=-8), A.AQ_ERR_INVALID_ARGUMENT, "features"),
    (dict(dtype=A.AQ_I8), A.AQ_ERR_INVALID_ARGUMENT, "dtype"),
    (dict(max_tokens=0), A.AQ_ERR_INVALID_ARGUMENT, "max_tokens"),
    (dict(dtype=A.AQ_F32), A.AQ_ERR_UNSUPPORTED, "fp16 or bf16"),
    (dict(features=60), A.AQ_ERR_UNSUPPORTED, "multiple of 8"),
    (dict(vocab=(1 << 30) + 1), A.AQ_ERR_UNSUPPORTED, "vocab"),
    (dict(max_tokens=(1 << 24) + 1), A.AQ_ERR_UNSUPPORTED, "max_tokens"),
    (dict(features=(1 << 21) + 8), A.AQ_ERR_UNSUPPORTED, "features"),
    (dict(max_tokens=(1 << 21) + 1), A.AQ_ERR_UNSUPPORTED, "max_tokens"),
])
def test_loss_create_refuses(change, status, text):
    st, h, msg = _create_loss(**change)
    assert st == status and text in msg and h is None


def test_null_handles():
    lib = _lib()
    assert lib.aq_usq_create(None, 16, 16, None, None) == A.AQ_ERR_INVALID_ARGUMENT
    assert lib.aq_usq_forward(None, 16, 16, 1, None) == A.AQ_ERR_INVALID_ARGUMENT
    assert lib.aq_usq_input_grad(None, 16, 16, 1, None) == A.AQ_ERR_INVALID_ARGUMENT
    assert lib.aq_usq_destroy(None) == A.AQ_OK
    assert lib.aq_loss_create(None, None) == A.AQ_ERR_INVALID_ARGUMENT
    assert lib.aq_loss_cross_entropy(None, 16, 16, 16, None, 16, None, None, 1, None) == A.AQ_ERR_INVALID_ARGUMENT
    assert lib.aq_loss_distill(None, 16, 16, 16, 1, 1.0, None, 16, None, 1, None) == A.AQ_ERR_INVALID_ARGUMENT
    assert lib.aq_loss_destroy(None) == A.AQ_OK


# ---- calls on a handle (in a child whose HIP calls go to host memory) ----

def usq_calls():
    st, h, msg = _create_usq()
    assert st == A.AQ_OK, msg
    lib, out = _lib(), []
    for name in ("aq_usq_forward", "aq_usq_input_grad"):
        f = getattr(lib, name)
        for args in ((None, 4096, 1), (4096, None, 1), (4096, 4096, 0), (4096, 4096, 9), (4104, 4096, 1), (4096, 4098, 1),
                     (4096, 4096, 8)):
            st = f(h, *args, None)
            out.append((st, lib.aq_last_error().decode() if st else ""))
    live = host_device.live_bytes()
    lib.aq_usq_destroy(h)
    return out, live, host_device.live_bytes()


def loss_calls():
    lib, out = _lib(), []
    _, h, msg = _create_loss()
    assert h, msg
    _, plain, _ = _create_loss(features=0, dtype=A.AQ_F32)
    P = 4096

    def ce(X=P, W=P, targets=P, dloss=2 * P, loss=P, dX=P, dW=P, n=1, on=h):
        return lib.aq_loss_cross_entropy(on, X, W, targets, dloss, loss, dX, dW, n, None)

    def di(logits=P, ids=P, teacher=P, top=2, T=1.0, dloss=P, loss=P, dlogits=P, n=1, on=h):
        return lib.aq_loss_distill(on, logits, ids, teacher, top, T, dloss, loss, dlogits, n, None)

    for f, kws in ((ce, [dict(X=None), dict(W=None), dict(targets=None), dict(loss=None), dict(n=0), dict(n=9),
                         dict(X=P + 2), dict(W=P + 8), dict(dX=P + 4), dict(dW=P + 8), dict(targets=P + 4),
                         dict(dloss=P + 2), dict(loss=P + 1), dict(on=plain), dict(dloss=P), dict(dloss=P + 28, n=8),
                         dict(dloss=P - 28, n=8), dict(dloss=P + 32, n=8), {},
                         dict(dX=None, dW=None, dloss=None, n=8)]),
                   (di, [dict(logits=None), dict(ids=None), dict(teacher=None), dict(loss=None), dict(n=0), dict(n=9),
                         dict(top=0), dict(top=1025), dict(T=0.0), dict(T=-1.0), dict(T=float("inf")),
                         dict(T=float("nan")), dict(logits=P + 8), dict(dlogits=P + 2), dict(ids=P + 2),
                         dict(teacher=P + 1), dict(teacher=P + 2, on=plain), {}, dict(on=plain, dlogits=None, dloss=None)])):
        for kw in kws:
            st = f(**kw)
            out.append((st, lib.aq_last_error().decode() if st else ""))
    lib.aq_loss_destroy(h)
    lib.aq_loss_destroy(plain)
    return out, host_device.live_bytes()


def launch_limits(n, features, vocab, top):
    """Statuses of calls of the given sizes: every launch is checked against the launch limits."""
    lib = _lib()
    _, h, msg = _create_loss(vocab=vocab, features=features, max_tokens=n)
    assert h, msg
    P = 4096
    got = [lib.aq_loss_cross_entropy(h, P, P, P, None, P, P, P, n, None),
           lib.aq_loss_distill(h, P, P, P, top, 1.0, None, P, P, n, None)]
    lib.aq_loss_destroy(h)
    return got


def usq_limits(n, K, C_out):
    lib = _lib()
    d = A.aq_usq_desc(C_out, K, 128, A.AQ_BF16, A.AQ_BF16, n)
    codes, h = np.zeros((C_out, K // 2), np.uint8), ctypes.c_void_p()
    scales = np.zeros((C_out, -(-K // 128)), np.uint16)
    assert lib.aq_usq_create(ctypes.byref(d), codes.ctypes.data, scales.ctypes.data, None, ctypes.byref(h)) == A.AQ_OK
    got = [lib.aq_usq_forward(h, 4096, 4096, n, None), lib.aq_usq_input_grad(h, 4096, 4096, n, None)]
    lib.aq_usq_destroy(h)
    return got


def usq_one_group():
    """Creation and calls of a layer whose group is the largest there is: one scale a row."""
    lib = _lib()
    live = host_device.live_bytes()
    st, h, msg = _create_usq(group=(1 << 31) - 128)
    assert st == A.AQ_OK, msg
    got = [host_device.live_bytes() - live, lib.aq_usq_forward(h, 4096, 4096, 1, None), lib.aq_usq_input_grad(h, 4096, 4096, 1, None)]
    lib.aq_usq_destroy(h)
    return got


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    _lib()
    return host_device.build(tmp_path_factory)


def test_usq_calls_refuse(so):
    out, live, left = host_device.in_child(so, "test_usq_losses_host", "usq_calls")
    texts = ["null", "null", "n must be", "max_tokens", "16-byte", "16-byte", ""] * 2
    assert [s for s, _ in out] == [A.AQ_ERR_INVALID_ARGUMENT if t else A.AQ_OK for t in texts]
    assert all(t in msg for t, (_, msg) in zip(texts, out))
    assert live > 0 and left == 0


def test_loss_calls_refuse(so):
    out, left = host_device.in_child(so, "test_usq_losses_host", "loss_calls")
    I, S = A.AQ_ERR_INVALID_ARGUMENT, A.AQ_ERR_UNSUPPORTED
    want = [(I, "null")] * 4 + [(I, "n must be"), (I, "max_tokens")] + [(I, "16-byte")] * 4 + [
        (I, "8-byte"), (I, "4-byte"), (I, "4-byte"), (I, "without features")] + [
        (I, "overlaps")] * 3 + [(0, "")] * 3
    want += [(I, "null")] * 4 + [(I, "n must be"), (I, "max_tokens"), (I, "top"), (S, "top")] + [(I, "temperature")] * 4 + [
        (I, "16-byte"), (I, "16-byte"), (I, "aligned"), (I, "aligned"), (I, "aligned"), (0, ""), (0, "")]
    assert [s for s, _ in out] == [s for s, _ in want]
    assert all(t in msg for (_, t), (_, msg) in zip(want, out))
    assert left == 0


def test_usq_largest_group(so):
    held, *got = host_device.in_child(so, "test_usq_losses_host", "usq_one_group")
    assert got == [0, 0] and held < 1 << 20


@pytest.mark.parametrize("n,features,vocab,top", [(1, 8, 1, 1), (70000, 64, 1000, 5), (3, 8, 3000000, 1024), (1 << 21, 8, 9, 1),
                                                    (257, 1 << 21, 300, 3)])
def test_loss_launches_stay_in_limits(so, n, features, vocab, top):
    assert host_device.in_child(so, "test_usq_losses_host", "launch_limits", n, features, vocab, top) == [0, 0]


@pytest.mark.parametrize("n,K,C_out", [(1, 8, 1), (1 << 24, 8, 3), (100, 128, 1100001), (1100000, 1152, 33), (1, 1 << 20, 1)])
def test_usq_launches_stay_in_limits(so, n, K, C_out):
    assert host_device.in_child(so, "test_usq_losses_host", "usq_limits", n, K, C_out) == [0, 0]


# ---- the binding's checks of tensors ----

@pytest.fixture
def host_tensors(monkeypatch):
    monkeypatch.setattr(A, "_DEVICE_TYPE", "cpu")


def _usq_shell():
    obj = object.__new__(A.USQLayer)
    obj.C_out, obj.K, obj.group, obj.dtype, obj.y_dtype, obj.device, obj.handle = C_OUT, K, 32, "f16", "f32", None, None
    return obj


def _loss_shell(dtype="f16", features=F):
    obj = object.__new__(A.VocabLoss)
    obj.vocab, obj.features, obj.dtype, obj.device, obj.handle = VOCAB, features, dtype, None, None
    return obj


@pytest.mark.parametrize("kw, text", [
    (dict(codes=np.zeros((C_OUT, K // 2), np.int8)), "codes must have dtype"),
    (dict(codes=np.zeros(5, np.uint8)), "matrix"),
    (dict(scales=np.ones((C_OUT, 2), np.float32)), "scales must have dtype"),
    (dict(scales=np.ones((C_OUT, 3), np.float16)), "scales must have shape"),
    (dict(zeros=np.ones((C_OUT, 2), np.int32)), "zeros must have dtype"),
    (dict(zeros=np.ones((2, C_OUT), np.uint8)), "zeros must have shape"),
    (dict(group=0), "group"),
    (dict(dtype="f32"), "dtype"),
    (dict(y_dtype="i8"), "y_dtype"),
])
def test_usq_layer_rejects_bad_arrays(kw, text):
    args = dict(codes=np.zeros((C_OUT, K // 2), np.uint8), scales=np.ones((C_OUT, 2), np.float16), zeros=None, group=32)
    args.update(kw)
    with pytest.raises(ValueError, match=text):
        A.USQLayer(args.pop("codes"), args.pop("scales"), args.pop("zeros"), max_tokens=4, **args)


def test_usq_tensor_checks(host_tensors):
    lay = _usq_shell()
    x = torch.zeros(3, K, dtype=torch.float16)
    for bad, text in ((x.float(), "dtype"), (x[:, :8].contiguous(), "shape"), (torch.zeros(3, 2 * K).half()[:, ::2], "contiguous"),
                      (x[:0], "at least one row"), (x[0], "matrix"), (x.numpy(), "matrix")):
        with pytest.raises(ValueError, match=text):
            lay.forward(bad)
    with pytest.raises(ValueError, match="out must have dtype"):
        lay.forward(x, out=torch.zeros(3, C_OUT).half())
    with pytest.raises(ValueError, match="out must have shape"):
        lay.forward(x, out=torch.zeros(2, C_OUT))
    with pytest.raises(ValueError, match="dy must have shape"):
        lay.input_grad(x)
    with pytest.raises(ValueError, match="out must have dtype"):
        lay.input_grad(torch.zeros(3, C_OUT).half(), out=torch.zeros(3, K))


def test_loss_tensor_checks(host_tensors):
    L = _loss_shell()
    x, w, t = torch.zeros(3, F).half(), torch.zeros(VOCAB, F).half(), torch.zeros(3, dtype=torch.int64)
    for kw, text in ((dict(x=x.float()), "x must have dtype"), (dict(x=x[:0]), "at least one row"),
                     (dict(w=w[:-1]), "w must have shape"), (dict(w=torch.zeros(F, VOCAB).half().t()), "w must be contiguous"),
                     (dict(targets=t.int()), "targets must have dtype"), (dict(targets=t[:2]), "targets must have shape"),
                     (dict(dloss=torch.zeros(3).half()), "dloss must have dtype"), (dict(loss=torch.zeros(4)), "loss must have shape"),
                     (dict(dx=torch.zeros(3, F)), "dx must have dtype"), (dict(dw=torch.zeros(F, VOCAB).half()), "dw must have shape")):
        args = dict(x=x, w=w, targets=t)
        args.update(kw)
        with pytest.raises(ValueError, match=text):
            L.cross_entropy(**args)
    with pytest.raises(ValueError, match="without features"):
        _loss_shell(features=None).cross_entropy(x, w, t)
    z, ids, te = torch.zeros(3, VOCAB).half(), torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, 5).half()
    for kw, text in ((dict(logits=z.float()), "logits must have dtype"), (dict(ids=ids.long()), "ids must have dtype"),
                     (dict(ids=ids[:, :0]), "at least one column"), (dict(ids=ids[:2]), "ids must have shape"),
                     (dict(teacher=te[:, :4].contiguous()), "teacher must have shape"), (dict(teacher=te.float()), "teacher must have dtype"),
                     (dict(grad=z.float()), "grad must have dtype")):
        args = dict(logits=z, ids=ids, teacher=te)
        args.update(kw)
        with pytest.raises(ValueError, match=text):
            L.distill(**args)


def test_descriptors_refuse_what_would_wrap():
    with pytest.raises(ValueError, match="2\\^31"):
        A.USQLayer(np.zeros((C_OUT, K // 2), np.uint8), np.ones((C_OUT, 1), np.float16), group=(1 << 32) + 32, max_tokens=4)
    with pytest.raises(ValueError, match="2\\^31"):
        A.VocabLoss((1 << 32) + 5, max_tokens=2)
    with pytest.raises(ValueError, match="2\\^31"):
        A.VocabLoss(5, features=(1 << 32) + 8, max_tokens=2)


@pytest.mark.parametrize("kw", [dict(dtype="i8"), dict(features=0)])
def test_vocab_loss_rejects(kw):
    with pytest.raises(ValueError):
        A.VocabLoss(VOCAB, max_tokens=2, **kw)
