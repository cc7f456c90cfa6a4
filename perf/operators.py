"""Operator cases: 4-bit layers with group scales, and the losses that a low-bit language model is tuned with.

A case is a dict of plain values; ``op`` names the operator:

* ``"usq"``: Y = X W^T of a linear layer whose weights are 4-bit codes with one scale (and zero point) per group of
  inputs, W[i][k] = s[i][k / group] * (q[i][k] - z[i][k / group]); single tokens, batches of tokens and prompts;
* ``"usq_grad"``: the same layer's input gradient dX = dY W;
* ``"distill"``: the distillation loss of student logits against a teacher's top logits, and its gradient;
* ``"cross_entropy"``: softmax cross entropy of a head's logits X W^T over a large vocabulary that keeps no logits,
  alone (``grads`` "none"), with the input gradient ("x") or with the input's and the head weights' ("xw").

``own`` is False: ``run`` computes the plain forms with elementary torch operations in 32 bits.  ``own`` is True: it
calls this package.  The ranges the listed cases stand for are those of ``draw``.
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _usq(name, n, K, C_out, group, dtype="f16", y=None, zeros=False, op="usq"):
    return {"name": name, "op": op, "n": n, "K": K, "C_out": C_out, "group": group, "dtype": dtype, "y": y or dtype,
            "zeros": zeros}


def _distill(name, n, vocab, top, dtype, T=1.0):
    return {"name": name, "op": "distill", "n": n, "vocab": vocab, "top": top, "dtype": dtype, "T": T}


def _ce(name, n, K, vocab, dtype, grads="xw"):
    return {"name": name, "op": "cross_entropy", "n": n, "K": K, "vocab": vocab, "dtype": dtype, "grads": grads}


def listed():
    return [
        # the smallest call: one token through an attention projection of the smallest width
        _usq("usq_token_small", 1, 576, 1728, 64),
        # one token being generated, a wide feed-forward layer: the whole time is the weights' read
        _usq("usq_token_wide", 1, 4096, 16384, 128, "bf16"),
        # a batch of sequences that generate together, odd output count, zero points, fine groups
        _usq("usq_batch", 23, 2304, 4999, 32, "f16", "f32", zeros=True),
        # a prompt
        _usq("usq_prompt", 4096, 4096, 4096, 128, "bf16"),
        # the gradient through a small frozen layer, a token count that fills no tile evenly
        _usq("usq_grad_small", 200, 1152, 576, 64, "f16", zeros=True, op="usq_grad"),
        # the gradient of a training batch through a wide frozen layer
        _usq("usq_grad_wide", 4096, 4096, 8192, 128, "bf16", op="usq_grad"),
        # distillation on a handful of positions
        _distill("distill_few", 4, 32768, 16, "f32"),
        # a batch over an odd vocabulary, softened teacher
        _distill("distill_odd", 1024, 49999, 50, "f16", 2.0),
        # a training batch over a large vocabulary
        _distill("distill_large", 4096, 131072, 64, "bf16"),
        # a small head, odd vocabulary, with both gradients
        _ce("ce_small", 100, 576, 4999, "f16"),
        # perplexity of held-out text: the loss alone
        _ce("ce_eval", 2048, 1024, 50021, "bf16", "none"),
        # a training batch over a large vocabulary, with both gradients
        _ce("ce_large", 4096, 4096, 131072, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_usq(rng):
    op = rng.choice(["usq", "usq", "usq_grad"])
    n = _log_int(rng, 1, 8192)
    if op == "usq" and rng.random() < 0.4:
        n = _log_int(rng, 1, 64)
    K = 8 * _log_int(rng, 16, 2048)
    C_out = _log_int(rng, 64, 16384)
    if rng.random() < 0.6:
        K, C_out = max(128, K // 128 * 128), max(64, C_out // 64 * 64)
    n = max(1, min(n, int(1.3e11 / (2.0 * K * C_out))))
    dtype = rng.choice(["f16", "bf16"])
    y = "f32" if op == "usq" and rng.random() < 0.25 else dtype
    return _usq("", n, K, C_out, rng.choice([32, 64, 128, 128, 256]), dtype, y, rng.random() < 0.5, op)


def _draw_distill(rng):
    vocab = _log_int(rng, 1000, 160000)
    n = max(1, min(_log_int(rng, 1, 8192), 4096 * 131072 // vocab))
    return _distill("", n, vocab, _log_int(rng, 1, 128), rng.choice(["f32", "f16", "bf16", "bf16"]),
                    rng.choice([1.0, 1.0, 2.0, 0.7]))


def _draw_ce(rng):
    K = 8 * _log_int(rng, 8, 512)
    vocab = _log_int(rng, 500, 131072)
    n = max(1, min(_log_int(rng, 1, 8192), int(2.0e12 / (2.0 * K * vocab))))
    return _ce("", n, K, vocab, rng.choice(["f16", "bf16", "bf16"]), rng.choice(["none", "x", "xw", "xw"]))


def draw(rng):
    r = rng.random()
    case = _draw_usq(rng) if r < 0.5 else _draw_distill(rng) if r < 0.75 else _draw_ce(rng)
    del case["name"]
    return case


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


def _usq_inputs(case, seed):
    """Bell-shaped codes around their zero point, packed two to a byte (the lower half first); scales that keep unit
    inputs at unit scale; activations with a few large channels, or output gradients of a mean's scale."""
    g = _gen(seed)
    n, K, C_out, group = case["n"], case["K"], case["C_out"], case["group"]
    G = -(-K // group)
    zeros = torch.randint(5, 12, (C_out, G), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    centre = 8.0 if zeros is None else zeros.float().repeat_interleave(group, 1)[:, :K]
    q = (_randn(g, C_out, K) * 2.7 + centre).round().clamp_(0, 15).to(torch.uint8)
    codes = q[:, 0::2] | (q[:, 1::2] << 4)
    del q, centre
    scales = ((_rand(g, C_out, G) + 0.5) / (2.8 * math.sqrt(K))).to(_TORCH[case["dtype"]])
    if case["op"] == "usq":
        x = _randn(g, n, K) * torch.where(_rand(g, K) < 0.01, 8.0, 1.0)
    else:
        x = _randn(g, n, C_out) * 0.1
    return codes.contiguous(), scales, zeros, x.to(_TORCH[case["dtype"]])


def _distill_inputs(case, seed):
    """Student logits of a spread of some three units; the teacher's largest logits at tokens the student mostly
    ranks high too, a few lists short (id -1 ends them), a few rows with no list at all."""
    g = _gen(seed)
    n, V, top = case["n"], case["vocab"], min(case["top"], case["vocab"])
    z = _randn(g, n, V) * 2.5
    near = _randn(g, n, 1).expand(n, V) if top == V else None
    score = z + 1.5 * _randn(g, n, V) if near is None else z + near
    t, ids = score.topk(top, dim=1)
    del score
    short = (_rand(g, n, 1) < 0.1) & (torch.arange(top, device="cuda")[None] >= (top + 1) // 2)
    none = _rand(g, n, 1) < 0.02
    ids = torch.where(short | none, -1, ids).to(torch.int32)
    dloss = (_rand(g, n) + 0.5) * (1024.0 if case["dtype"] == "f16" else 1.0) / n
    return z.to(_TORCH[case["dtype"]]), ids.contiguous(), t.to(_TORCH[case["dtype"]]).contiguous(), dloss


def _ce_inputs(case, seed):
    """Hidden states, a head whose row of the target token leans towards them (a model that has learned something),
    and next tokens, some positions (-1) not counted.  An fp16 program scales its loss."""
    g = _gen(seed)
    n, K, V = case["n"], case["K"], case["vocab"]
    dt = _TORCH[case["dtype"]]
    x = _randn(g, n, K)
    w = _randn(g, V, K) * (2.0 / math.sqrt(K))
    targets = torch.randint(0, V, (n,), generator=g, device="cuda")
    x += 0.5 * _rand(g, n, 1) * math.sqrt(K) * w[targets]
    targets = torch.where(_rand(g, n) < 0.05, -1, targets)
    dloss = torch.full((n,), (1024.0 if case["dtype"] == "f16" else 1.0) / n, device="cuda")
    return x.to(dt), w.to(dt), targets, dloss


def prepare(case, seed):
    op, dt = case["op"], _TORCH[case["dtype"]]
    state = dict(case)
    if op in ("usq", "usq_grad"):
        codes, scales, zeros, x = _usq_inputs(case, seed)
        state.update(codes=codes, scales=scales, zero_points=zeros, x=x)
        state["out"] = torch.empty((case["n"], case["C_out"] if op == "usq" else case["K"]),
                                   dtype=_TORCH[case["y"]] if op == "usq" else dt, device="cuda")
        if own:
            import paper_2506_05960_amd as aq
            state["layer"] = aq.USQLayer(codes.cpu(), scales.cpu(), None if zeros is None else zeros.cpu(),
                                         group=case["group"], dtype=case["dtype"], y_dtype=case["y"],
                                         max_tokens=case["n"])
        return state
    if op == "distill":
        z, ids, t, dloss = _distill_inputs(case, seed)
        state.update(z=z, ids=ids, t=t, dloss=dloss, loss=torch.empty(case["n"], device="cuda"),
                     grad=torch.empty_like(z))
    else:
        x, w, targets, dloss = _ce_inputs(case, seed)
        state.update(x=x, w=w, targets=targets, dloss=dloss, loss=torch.empty(case["n"], device="cuda"),
                     dx=torch.empty_like(x) if "x" in case["grads"] else None,
                     dw=torch.empty_like(w) if "w" in case["grads"] else None)
    if own:
        import paper_2506_05960_amd as aq
        state["losses"] = aq.VocabLoss(case["vocab"], features=case.get("K"), dtype=case["dtype"],
                                       max_tokens=case["n"])
    return state


# ---- one pass ----

def _run_own(s):
    if s["op"] == "usq":
        return s["layer"].forward(s["x"], out=s["out"])
    if s["op"] == "usq_grad":
        return s["layer"].input_grad(s["x"], out=s["out"])
    if s["op"] == "distill":
        return s["losses"].distill(s["z"], s["ids"], s["t"], temperature=s["T"], dloss=s["dloss"], loss=s["loss"],
                                   grad=s["grad"])
    got = s["losses"].cross_entropy(s["x"], s["w"], s["targets"], dloss=s["dloss"], loss=s["loss"], dx=s["dx"],
                                    dw=s["dw"])
    return [v for v in got if v is not None]


def _dequantized(s):
    """The layer's weights in 32 bits."""
    codes, group = s["codes"], s["group"]
    q = torch.stack([codes & 15, codes >> 4], dim=2).reshape(s["C_out"], s["K"]).float()
    scales = s["scales"].float().repeat_interleave(group, 1)[:, :s["K"]]
    zeros = 8.0 if s["zero_points"] is None else s["zero_points"].float().repeat_interleave(group, 1)[:, :s["K"]]
    return (q - zeros) * scales


def _run_usq(s):
    w = _dequantized(s)
    return (s["x"].float() @ (w.t() if s["op"] == "usq" else w)).to(s["out"].dtype)


def _run_distill(s):
    T = s["T"]
    z, listed_ = s["z"].float() / T, s["ids"] >= 0
    top = z.amax(dim=1, keepdim=True)
    q = torch.exp(z - top)
    total = q.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    q /= total
    counts = listed_.any(dim=1, keepdim=True)
    t = torch.where(listed_, s["t"].float() / T, -math.inf)
    t = t - torch.where(counts, t.amax(dim=1, keepdim=True), 0.0)
    p = torch.exp(t)
    mass = torch.where(counts, p.sum(dim=1, keepdim=True), 1.0)
    p = p / mass
    at = s["ids"].clamp(min=0).long()
    terms = torch.where(p > 0, p * (t - torch.log(mass) - (z.gather(1, at) - lse)), 0.0)
    loss = T * T * terms.sum(dim=1)
    grad = q.scatter_add_(1, at, -p)
    grad *= (T * s["dloss"])[:, None] * counts
    return loss, grad.to(s["z"].dtype)


def _run_ce(s):
    x, w, counted = s["x"].float(), s["w"].float(), s["targets"] >= 0
    z = x @ w.t()
    top = z.amax(dim=1, keepdim=True)
    at = s["targets"].clamp(min=0)[:, None]
    hit = z.gather(1, at)
    p = torch.exp(z - top)
    del z
    total = p.sum(dim=1, keepdim=True)
    loss = torch.where(counted, (top + torch.log(total) - hit)[:, 0], 0.0)
    if s["grads"] == "none":
        return [loss]
    p /= total
    p.scatter_add_(1, at, torch.full_like(hit, -1.0))
    p *= (s["dloss"] * counted)[:, None]
    dx = (p @ w).to(s["x"].dtype)
    if s["grads"] == "x":
        return [loss, dx]
    return [loss, dx, (p.t() @ x).to(s["w"].dtype)]


def run(state):
    if own:
        return _run_own(state)
    if state["op"] in ("usq", "usq_grad"):
        return _run_usq(state)
    return _run_distill(state) if state["op"] == "distill" else _run_ce(state)


# ---- what a pass cannot do without ----

def work(case):
    n, b = case["n"], _BYTES[case["dtype"]]
    if case["op"] in ("usq", "usq_grad"):
        K, C_out = case["K"], case["C_out"]
        G = -(-K // case["group"])
        weights = C_out * K // 2 + C_out * G * (b + (0.5 if case["zeros"] else 0))
        data = n * K * b + n * C_out * _BYTES[case["y"]]
        return {"bytes": weights + data, "flops": 2.0 * n * K * C_out}
    if case["op"] == "distill":
        V, top = case["vocab"], min(case["top"], case["vocab"])
        # logits in, gradient out, the lists, row weights and losses; an exponential and some four operations a logit
        return {"bytes": 2 * n * V * b + n * top * (4 + b) + 8 * n, "flops": 5.0 * n * V}
    K, V = case["K"], case["vocab"]
    products = {"none": 1, "x": 2, "xw": 3}[case["grads"]]     # the logits' product, and one for each gradient
    data = (n * K + V * K) * b + 16 * n
    data += n * K * b * ("x" in case["grads"]) + V * K * b * ("w" in case["grads"])
    return {"bytes": data, "flops": 2.0 * n * K * V * products}


# ---- the same in 64 bits, from the definitions ----

def _exact_usq(case, seed):
    codes, scales, zeros, x = _usq_inputs(case, seed)
    C_out, K = case["C_out"], case["K"]
    w = torch.empty((C_out, K), dtype=torch.float64, device="cuda")
    w[:, 0::2] = (codes % 16).double()
    w[:, 1::2] = (codes // 16).double()
    j = torch.arange(K, device="cuda") // case["group"]
    w -= zeros.double()[:, j] if zeros is not None else 8
    w *= scales.double()[:, j]
    return torch.matmul(x.double(), w.T if case["op"] == "usq" else w)


def _exact_distill(case, seed):
    z, ids, t, dloss = _distill_inputs(case, seed)
    T = case["T"]
    log_q = torch.log_softmax(z.double() / T, dim=1)
    log_p = torch.log_softmax((t.double() / T).masked_fill(ids < 0, -1e300), dim=1)
    counts = (ids >= 0).sum(dim=1) > 0
    log_p = log_p.masked_fill(ids < 0, -math.inf)
    log_p[~counts] = -math.inf
    p = log_p.exp()
    rows = torch.arange(case["n"], device="cuda")[:, None].expand_as(p)[ids >= 0]
    cols = ids[ids >= 0].long()
    loss = torch.zeros(case["n"], dtype=torch.float64, device="cuda")
    loss.index_add_(0, rows, p[ids >= 0] * (log_p[ids >= 0] - log_q[rows, cols]))
    grad = log_q.exp_()
    grad[rows, cols] -= p[ids >= 0]
    grad *= torch.where(counts, T * dloss.double(), 0.0)[:, None]
    return loss * T * T, grad


def _exact_ce(case, seed):
    x, w, targets, dloss = _ce_inputs(case, seed)
    x, w = x.double(), w.double()
    log_p = torch.log_softmax(x @ w.T, dim=1)
    rows = torch.arange(case["n"], device="cuda")[targets >= 0]
    cols = targets[targets >= 0]
    loss = torch.zeros(case["n"], dtype=torch.float64, device="cuda")
    loss[rows] = -log_p[rows, cols]
    if case["grads"] == "none":
        return [loss]
    p = log_p.exp_()
    p[rows, cols] -= 1
    p *= torch.where(targets >= 0, dloss.double(), 0.0)[:, None]
    return [loss, p @ w] if case["grads"] == "x" else [loss, p @ w, p.T @ x]


def exact(case, seed):
    if case["op"] in ("usq", "usq_grad"):
        return _exact_usq(case, seed)
    return _exact_distill(case, seed) if case["op"] == "distill" else _exact_ce(case, seed)
