"""Measured cases of the training losses.

Two operators, each in both directions:

* the cross entropy of a vocabulary head (``trimmoe_head_cross_entropy`` and
  its ``_backward``): for rows h_t, a head w [V, d] with bias b and targets y,
  loss_t = logsumexp_v(z_tv) - z_{t, y_t} with z = h w^T + b, and the gradients
  of sum_t g_t loss_t in h, w and b.  A target outside [0, V) takes no part;
* the balance loss of a router (``trimmoe_balance_loss`` and its
  ``_backward``): p_t = softmax(w h_t + b), counts c_e of the routed slots,
  S of them in n rows, L = E / (S n) * sum_e c_e * sum_t p_te, and its
  gradients with the counts held constant.  Slots of -1 are not routed; a row
  without a routed slot takes no part.

``listed`` holds the head and router shapes that the framework's workloads
name (the tiny, Switch-Base, Qwen-MoE and Mixtral layers) at batches from one
decode step to a prefill; ``draw`` spreads over the same ranges.  All inputs
are made on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"

# d_model, vocabulary, experts, routed slots of the workloads' layers
SHAPES = {
    "tiny": dict(d=64, vocab=512, experts=8, top_k=1),
    "switch": dict(d=768, vocab=32128, experts=8, top_k=1),
    "qwen": dict(d=2048, vocab=151936, experts=60, top_k=4),
    "mixtral": dict(d=4096, vocab=32000, experts=8, top_k=2),
}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _head(name, kind, shape, rows, dtype="bf16", bias=False, ignored=0.0, **over):
    s = dict(SHAPES[shape], **over)
    c = dict(kind=kind, d=s["d"], vocab=s["vocab"], rows=rows, dtype=dtype, bias=bias,
             ignored=ignored)
    return dict(c, name=name) if name else c


def _balance(name, kind, shape, rows, dtype="bf16", inactive=0.0, **over):
    s = dict(SHAPES[shape], **over)
    c = dict(kind=kind, d=s["d"], experts=s["experts"], top_k=s["top_k"], rows=rows, dtype=dtype,
             inactive=inactive)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest head: one request's 64 tokens scored, fp32; latency
        _head("head_loss_tiny_f32_64", "head_loss", "tiny", 64, "f32", bias=True),
        # scoring one decode batch against the Mixtral vocabulary: W is read once
        _head("head_loss_mixtral_32", "head_loss", "mixtral", 32),
        # held-out loss of a prefill batch
        _head("head_loss_mixtral_8192", "head_loss", "mixtral", 8192, ignored=0.05),
        # one odd, short sample's gradient on the smallest head; latency
        _head("head_grad_tiny_37", "head_grad", "tiny", 37, bias=True),
        # a few tokens adapt a large head online: W read, dW written
        _head("head_grad_mixtral_16", "head_grad", "mixtral", 16),
        # the Switch-Base batch, short rows, a bias, prompt tokens ignored
        _head("head_grad_switch_4096", "head_grad", "switch", 4096, bias=True, ignored=0.3),
        # a ragged micro-batch against the largest vocabulary
        _head("head_grad_qwen_2047", "head_grad", "qwen", 2047, ignored=0.05),
        # the Mixtral batch: the largest products
        _head("head_grad_mixtral_8192", "head_grad", "mixtral", 8192, ignored=0.05),
        # fp32 storage at the Switch-Base shape
        _head("head_grad_switch_f32_777", "head_grad", "switch", 777, "f32", bias=True),
        # routing of one short request watched and corrected, fp32; latency
        _balance("balance_step_tiny_f32_64", "balance_step", "tiny", 64, "f32", inactive=0.1),
        # the load of a Mixtral prefill batch, loss only
        _balance("balance_loss_mixtral_8192", "balance_loss", "mixtral", 8192),
        # a training step of a router over many experts, some tokens exited early
        _balance("balance_step_qwen_8191", "balance_step", "qwen", 8191, inactive=0.2),
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["head_loss", "head_grad", "head_grad", "balance_loss", "balance_step"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind.startswith("head"):
        if rng.random() < 0.5:
            shape = rng.choice(["switch", "qwen", "mixtral"])
            d, vocab = SHAPES[shape]["d"], SHAPES[shape]["vocab"]
        else:
            d = 64 * _log_int(rng, 1, 64) if dtype == "bf16" else _log_int(rng, 40, 2048)
            vocab = _log_int(rng, 500, 60000)
        # no more than the largest listed case: rows x vocab x d (fp32 at a tenth of the rate)
        most = 8192 * 32000 * 4096 // (40 if dtype == "f32" else 1)
        rows = _log_int(rng, 1, max(1, min(8192, most // (d * vocab))))
        return _head(None, kind, "tiny", rows, dtype, bias=rng.random() < 0.5,
                     ignored=rng.choice([0.0, 0.05, 0.5]), d=d, vocab=vocab)
    if rng.random() < 0.5:
        shape = rng.choice(["switch", "qwen", "mixtral"])
        d, experts, top_k = (SHAPES[shape][n] for n in ("d", "experts", "top_k"))
    else:
        d = 64 * _log_int(rng, 1, 64) if dtype == "bf16" else _log_int(rng, 40, 4096)
        experts = _log_int(rng, 2, 256)
        top_k = rng.randint(1, min(8, experts))
    return _balance(None, kind, "tiny", _log_int(rng, 1, 8192), dtype,
                    inactive=rng.choice([0.0, 0.2]), d=d, experts=experts, top_k=top_k)


# ----------------------------------------------------------------- inputs --
def _randn(g, shape, sigma=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(sigma)


def _rand(g, shape):
    return torch.rand(shape, generator=g, device=DEV, dtype=torch.float32)


def _head_inputs(c, g):
    T, d, V, t = c["rows"], c["d"], c["vocab"], TYPES[c["dtype"]]
    w = _randn(g, (V, d), 1.0 / math.sqrt(d)).to(t)
    h = _randn(g, (T, d))
    target = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    # a partly trained head: rows lean towards their target by 0 to 12 logits
    wt = w[target.long()].float()
    h += wt * (12.0 * _rand(g, (T, 1)) / wt.square().sum(1, keepdim=True).clamp_min(1e-6))
    h = h.to(t)
    target[_rand(g, (T,)) < c["ignored"]] = -1
    b = _randn(g, (V,), 0.5) if c["bias"] else None
    s = dict(kind=c["kind"], w=w, h=h, b=b, target=target)
    if c["kind"] == "head_grad":
        # the mean over the rows that take part, and what the loss's call left
        s["dloss"] = (target >= 0).float() / (target >= 0).sum().clamp_min(1)
        z = torch.matmul(h.float(), w.float().t())
        s["lse"] = torch.logsumexp((z if b is None else z + b), 1)
    return s


def _balance_inputs(c, g):
    T, d, E, k, t = c["rows"], c["d"], c["experts"], c["top_k"], TYPES[c["dtype"]]
    w = _randn(g, (E, d), 1.0 / math.sqrt(d)).to(t)
    b = -0.5 * torch.log(torch.arange(1, E + 1, device=DEV, dtype=torch.float32))  # a skewed load
    h = _randn(g, (T, d)).to(t)
    z = torch.matmul(h.float(), w.float().t()) + b
    target = torch.topk(z, k, dim=1).indices.to(torch.int16)  # as a trace records it
    target[_rand(g, (T,)) < c["inactive"]] = -1
    return dict(kind=c["kind"], w=w, h=h, b=b, target=target,
                dloss=torch.full((1,), 0.01, device=DEV))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return (_head_inputs if case["kind"].startswith("head") else _balance_inputs)(case, g)


# -------------------------------------------------------------------- run --
def _plain_head_loss(s):
    z = torch.matmul(s["h"].float(), s["w"].float().t())
    if s["b"] is not None:
        z = z + s["b"]
    m = z.max(1, keepdim=True).values
    lse = (m + (z - m).exp().sum(1, keepdim=True).log()).squeeze(1)
    y = s["target"].long()
    zy = z.gather(1, y.clamp_min(0).unsqueeze(1)).squeeze(1)
    return dict(loss=torch.where(y >= 0, lse - zy, 0.0), lse=lse)


def _plain_head_grad(s):
    h, w, y = s["h"].float(), s["w"].float(), s["target"].long()
    z = torch.matmul(h, w.t())
    if s["b"] is not None:
        z = z + s["b"]
    dz = (z - s["lse"].unsqueeze(1)).exp()
    col = torch.arange(w.shape[0], device=DEV)
    dz = (dz - (col == y.unsqueeze(1)).float()) * torch.where(y >= 0, s["dloss"], 0.0).unsqueeze(1)
    out = dict(dh=torch.matmul(dz, w).to(s["h"].dtype), dw=torch.matmul(dz.t(), h).to(s["w"].dtype))
    if s["b"] is not None:
        out["db"] = dz.sum(0)
    return out


def _plain_balance(s, grad):
    h, w, t = s["h"].float(), s["w"].float(), s["target"].long()
    E = w.shape[0]
    z = torch.matmul(h, w.t()) + s["b"]
    e = (z - z.max(1, keepdim=True).values).exp()
    p = e / e.sum(1, keepdim=True)
    experts = torch.arange(E, device=DEV)
    live = (t >= 0).any(1)
    slots = (t.unsqueeze(2) == experts).sum((0, 1))
    n = live.sum()
    counts = torch.cat([slots, n.reshape(1)]).to(torch.int32)
    part = torch.where(live.unsqueeze(1), p, 0.0)
    prob_sum = part.sum(0)
    scale = E / (slots.sum().float() * n.float()).clamp_min(1.0)
    loss = (scale * (slots.float() * prob_sum).sum()).reshape(1)
    out = dict(loss=loss, counts=counts, prob_sum=prob_sum, prob=p)
    if grad:
        c = slots.float() - slots.float().mean()
        dz = s["dloss"] * scale * part * (c - (p * c).sum(1, keepdim=True))
        out |= dict(dh=torch.matmul(dz, w).to(s["h"].dtype),
                    dw=torch.matmul(dz.t(), h).to(s["w"].dtype), db=dz.sum(0))
    return out


def _own(s):
    from paper_2608_00573_amd import abi
    if s["kind"] == "head_loss":
        loss, lse = abi.trimmoe_head_cross_entropy(s["w"], s["h"], s["target"], s["b"])
        return dict(loss=loss, lse=lse)
    if s["kind"] == "head_grad":
        dh, dw, db = abi.trimmoe_head_cross_entropy_backward(s["w"], s["h"], s["target"], s["lse"],
                                                             s["dloss"], s["b"])
        return dict(dh=dh, dw=dw) if db is None else dict(dh=dh, dw=dw, db=db)
    loss, counts, prob_sum, prob = abi.trimmoe_balance_loss(s["w"], s["h"], s["target"], s["b"])
    out = dict(loss=loss, counts=counts, prob_sum=prob_sum, prob=prob)
    if s["kind"] == "balance_step":
        dh, dw, db = abi.trimmoe_balance_loss_backward(s["w"], s["h"], s["target"], prob, counts,
                                                       s["dloss"])
        out |= dict(dh=dh, dw=dw, db=db)
    return out


def run(state):
    if own:
        return _own(state)
    if state["kind"] == "head_loss":
        return _plain_head_loss(state)
    if state["kind"] == "head_grad":
        return _plain_head_grad(state)
    return _plain_balance(state, state["kind"] == "balance_step")


# ------------------------------------------------------------------- work --
def work(case):
    T, d, size = case["rows"], case["d"], TYPES[case["dtype"]].itemsize
    if case["kind"].startswith("head"):
        V = case["vocab"]
        bias = 4 * V if case["bias"] else 0
        if case["kind"] == "head_loss":
            return dict(bytes=(V + T) * d * size + bias + 12 * T, flops=2 * T * V * d)
        # logits again (they are not among the inputs), then both products
        return dict(bytes=2 * (V + T) * d * size + 2 * bias + 12 * T, flops=6 * T * V * d)
    E, k = case["experts"], case["top_k"]
    small = 4 * E + 2 * T * k + 4 * T * E + 8 * E
    if case["kind"] == "balance_loss":
        return dict(bytes=(E + T) * d * size + small, flops=2 * T * E * d)
    return dict(bytes=2 * (E + T) * d * size + small + 4 * E, flops=6 * T * E * d)


# ------------------------------------------------------------------ exact --
def exact(case, seed):
    s = prepare(case, seed)
    h, w = s["h"].double(), s["w"].double()
    z = h @ w.T
    if s["b"] is not None:
        z += s["b"].double()
    y = s["target"].long()
    if case["kind"] == "head_loss":
        lse = torch.logsumexp(z, 1)
        rows = torch.arange(z.shape[0], device=DEV)
        loss = lse - z[rows, y.clamp(min=0)]
        loss[y < 0] = 0
        return dict(loss=loss, lse=lse)
    if case["kind"] == "head_grad":
        # the gradient's value at the exact logits: softmax rows, one taken off at the target
        dz = torch.softmax(z, 1)
        del z
        rows = torch.nonzero(y >= 0).squeeze(1)
        dz[rows, y[rows]] -= 1
        g = s["dloss"].double()
        g[y < 0] = 0
        dz *= g[:, None]
        out = dict(dh=dz @ w, dw=dz.T @ h)
        if s["b"] is not None:
            out["db"] = dz.sum(0)
        return out
    E = w.shape[0]
    p = torch.softmax(z, 1)
    live = y.max(1).values >= 0
    slots = torch.bincount(y[y >= 0], minlength=E).double()
    n = float(live.sum())
    total = float(slots.sum())
    f = E * slots / (total * n) if n else slots
    prob_sum = p[live].sum(0)
    out = dict(loss=(f @ prob_sum).reshape(1), counts=None, prob_sum=prob_sum, prob=p)
    if case["kind"] == "balance_step":
        dz = float(s["dloss"]) * (p * f - p * (p @ f)[:, None])
        dz[~live] = 0
        out |= dict(dh=dz @ w, dw=dz.T @ h, db=dz.sum(0))
    return out
