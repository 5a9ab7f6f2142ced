"""Workloads of the operators around the convolution passes in a training step on discrete inputs:
what turns tokens into planes, what turns features into a loss, and what bounds the step.

A case is a dict.  `op` says which operator a pass goes through:

  embedding_fprop     rows (or planes) of a table by token, scaled
  embedding_accgrad   the gradient of that table from the gradient of its output
  xent_fprop          loss of a linear classifier over V classes and the log of its normaliser, by row
  xent_train          the same, then the gradients of the features and of the classifier's weights
  grad_norm           the 2-norm of many gradients taken together
  grad_clip           the same, and the gradients scaled so that it is at most max_norm

`type` is the type of the operands.  `T` = 0: features are rows [N, D].  `T` > 0: they are planes
[N / T, D, T], T positions in each of N / T samples, as the convolution passes take and give them.
A token or target outside 0 .. V-1 stands for no token: `kept` is the share of rows that have one.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_handle = None


def _hd():
    global _handle
    if _handle is None:
        import paper_1412_7580_amd as pkg
        _handle = pkg.Handle(0)
    return _handle


def _case(name, op, type, N, D, V, T=0, kept=1.0):
    return {"name": name, "op": op, "type": type, "N": N, "D": D, "V": V, "T": T, "kept": kept}


def _list(name, op, type, count, total, ratio):
    return {"name": name, "op": op, "type": type, "count": count, "total": total, "ratio": ratio}


def listed():
    return [
        # one position scored against a vocabulary: latency, one pass over the weights
        _case("score_1_bf16", "xent_fprop", "bf16", 1, 1024, 32000),
        # a short text scored, vocabulary of odd size
        _case("score_61_f16", "xent_fprop", "f16", 61, 768, 50001),
        # every position of a 13x13 layer's 11x11 outputs, 384 planes, classified into 1000 classes
        _case("train_planes_f32", "xent_train", "f32", 128 * 121, 384, 1000, T=121),
        # the ordinary training step of a model with a vocabulary
        _case("train_4096_bf16", "xent_train", "bf16", 4096, 1024, 32000),
        # a padded batch: a third of its rows have no target, sizes that no tile divides
        _case("train_padded_bf16", "xent_train", "bf16", 3001, 1000, 50001, kept=0.65),
        # the largest
        _case("train_8192_bf16", "xent_train", "bf16", 8192, 2048, 65536),
        # one token's row: latency
        _case("embed_1_bf16", "embedding_fprop", "bf16", 1, 1024, 32000),
        # 27x27 maps of tokens into the 64 planes of a convolution layer
        _case("embed_planes_f32", "embedding_fprop", "f32", 64 * 729, 64, 10007, T=729, kept=0.9),
        # the table's gradient in the ordinary training step
        _case("embed_grad_bf16", "embedding_accgrad", "bf16", 16384, 1024, 32000),
        # the table's gradient behind a convolution layer's gradient in planes
        _case("embed_grad_planes_f32", "embedding_accgrad", "f32", 128 * 729, 64, 10007, T=729, kept=0.9),
        # the gradients of a small net of convolution layers
        _list("norm_small_f32", "grad_norm", "f32", 12, 1_600_000, 1.0),
        # the gradients of a large net, clipped in a step whose norm is well above the limit
        _list("clip_large_bf16", "grad_clip", "bf16", 60, 400_000_000, 0.37),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embedding_fprop", "embedding_accgrad", "xent_fprop", "xent_train", "xent_train", "grad_norm", "grad_clip"])
    type = rng.choice(["f32", "bf16", "f16"])
    if op.startswith("grad"):
        return {"op": op, "type": type, "count": _log(rng, 1, 60), "total": _log(rng, 100, 200_000_000), "ratio": rng.choice([0.1, 0.37, 3.0])}
    kept = rng.choice([1.0, 1.0, 0.9, 0.5])
    T = _log(rng, 2, 729) if rng.random() < 0.3 else 0
    if op.startswith("embedding"):
        N, D, V = _log(rng, 1, 65536), _log(rng, 8, 1024), _log(rng, 2, 65536)
    else:
        N, D, V = _log(rng, 1, 8192), _log(rng, 16, 2048), _log(rng, 2, 65536)
        if type == "f32":
            N = min(N, 4096)
    if T:
        N = max(1, N // T) * T
    return {"op": op, "type": type, "N": N, "D": D, "V": V, "T": T, "kept": kept}


def _tokens(case, g):
    """Tokens as text has them: a token's share falls with its rank."""
    N, V = case["N"], case["V"]
    u = torch.rand(N, generator=g, device="cuda", dtype=torch.float64)
    t = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    if case["kept"] < 1.0:
        t[torch.rand(N, generator=g, device="cuda") >= case["kept"]] = -1
    return t.view(-1, case["T"]) if case["T"] else t


def _features(case, g, scale=1.0):
    N, D, T = case["N"], case["D"], case["T"]
    shape = (N // T, D, T) if T else (N, D)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(TYPES[case["type"]])


def _loss_scale(case):
    """The mean loss, in fp16 scaled as such training does: its gradients are below what that type holds."""
    return float(case["N"]) if case["type"] == "f16" else 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = TYPES[case["type"]]
    if case["op"].startswith("grad"):
        # sizes as a net has them: a few large matrices, many small vectors
        import random
        r = random.Random(1000003 * case["count"] + case["total"])
        share = [math.exp(r.uniform(-6.0, 0.0)) for _ in range(case["count"])]
        sizes = [max(1, int(case["total"] * s / sum(share))) for s in share]
        grads = [torch.randn(n, generator=g, device="cuda").mul_(0.02).to(dt) for n in sizes]
        state = {"case": case, "grads": grads, "max_norm": case["ratio"] * 0.02 * math.sqrt(sum(sizes))}
        if case["op"] == "grad_clip":
            state["out"] = [torch.empty_like(t) for t in grads]
        return state
    state = {"case": case, "tokens": _tokens(case, g)}
    if case["op"] == "embedding_fprop":
        state["table"] = torch.randn(case["V"], case["D"], generator=g, device="cuda").to(dt)
    elif case["op"] == "embedding_accgrad":
        state["gy"] = _features(case, g, 0.01)
    else:
        state["x"] = _features(case, g)
        state["wt"] = (torch.randn(case["V"], case["D"], generator=g, device="cuda") * (1.5 / math.sqrt(case["D"]))).to(dt)
    return state


def _rows(x, planes):
    """[N, D] from rows or planes."""
    return x.transpose(1, 2).reshape(-1, x.shape[1]) if planes else x


def _unrows(x, like):
    return x.view(like.shape[0], like.shape[2], like.shape[1]).transpose(1, 2).contiguous() if like.dim() == 3 else x


def run(state):
    case = state["case"]
    op, planes = case["op"], case.get("T", 0) > 0
    scale = math.sqrt(case["D"]) if op.startswith("embedding") else 1.0
    if own:
        hd = _hd()
        if op == "embedding_fprop":
            return hd.embedding_fprop(state["table"], state["tokens"], scale=scale, planes=planes)
        if op == "embedding_accgrad":
            return hd.embedding_accgrad(state["gy"], state["tokens"], case["V"], scale=scale, planes=planes)
        if op == "grad_norm":
            return hd.grad_norm(state["grads"])
        if op == "grad_clip":
            norm = hd.grad_clip(state["grads"], state["max_norm"], out=state["out"])
            return {"norm": norm, "out": state["out"]}
        x, wt, t = state["x"], state["wt"], state["tokens"]
        loss, lse = hd.xent_fprop(x, wt, t, planes=planes)
        if op == "xent_fprop":
            return {"loss": loss, "lse": lse}
        gx, gw = hd.xent_backward(x, wt, t, lse, scale=_loss_scale(case), mean=True, planes=planes)
        return {"loss": loss, "lse": lse, "gx": gx, "gw": gw}

    if op.startswith("grad"):
        total = torch.stack([t.float().square().sum() for t in state["grads"]]).sum()
        norm = total.sqrt()
        if op == "grad_norm":
            return norm
        c = torch.clamp(state["max_norm"] / norm, max=1.0)
        return {"norm": norm, "out": [(t.float() * c).to(t.dtype) for t in state["grads"]]}
    tokens = state["tokens"].reshape(-1)
    has = (tokens >= 0) & (tokens < case["V"])
    at = torch.where(has, tokens, torch.zeros_like(tokens))
    if op == "embedding_fprop":
        y = state["table"][at].float() * scale * has[:, None]
        y = y.to(state["table"].dtype)
        if planes:
            y = y.view(-1, case["T"], case["D"]).transpose(1, 2).contiguous()
        return y
    if op == "embedding_accgrad":
        gy = _rows(state["gy"], planes).float() * has[:, None]
        gt = torch.zeros(case["V"], case["D"], device=gy.device).index_add_(0, at, gy)
        return (gt * scale).to(state["gy"].dtype)
    x, wt = _rows(state["x"], planes).float(), state["wt"].float()
    logits = x @ wt.t()
    top = logits.amax(1, keepdim=True)
    lse = (logits - top).exp().sum(1, keepdim=True).log() + top
    loss = (lse - logits.gather(1, at[:, None])) * has[:, None]
    lse = lse * has[:, None]
    out = {"loss": loss.view(state["tokens"].shape), "lse": lse.view(state["tokens"].shape)}
    if op == "xent_train":
        p = (logits - lse).exp_()
        p.scatter_add_(1, at[:, None], torch.full_like(loss, -1.0))
        p *= has[:, None] * (_loss_scale(case) / has.sum().clamp(min=1))
        out["gx"] = _unrows((p @ wt).to(state["x"].dtype), state["x"])
        out["gw"] = (p.t() @ x).to(state["wt"].dtype)
    return out


def exact(case, seed):
    state = prepare(case, seed)
    op, T = case["op"], case.get("T", 0)
    if op.startswith("grad"):
        norm = math.sqrt(sum(float(torch.dot(t.double(), t.double())) for t in state["grads"]))
        if op == "grad_norm":
            return norm
        c = min(1.0, state["max_norm"] / norm) if norm else 1.0
        return {"norm": norm, "out": [t.double().mul_(c) for t in state["grads"]]}
    D, V = case["D"], case["V"]
    tokens = state["tokens"].flatten()
    kept = torch.nonzero((tokens >= 0) & (tokens < V)).flatten()
    t = tokens[kept]

    def to_rows(v):
        return v.double().permute(0, 2, 1).reshape(-1, D) if T else v.double()

    def from_rows(v):
        return v.reshape(-1, T, D).permute(0, 2, 1).contiguous() if T else v

    if op == "embedding_fprop":
        y = torch.zeros(case["N"], D, dtype=torch.float64, device="cuda")
        y[kept] = state["table"].double()[t] * math.sqrt(D)
        return from_rows(y)
    if op == "embedding_accgrad":
        gt = torch.zeros(V, D, dtype=torch.float64, device="cuda")
        gt.index_put_((t,), to_rows(state["gy"])[kept], accumulate=True)
        return gt * math.sqrt(D)
    x, w = to_rows(state["x"]), state["wt"].double()
    shape = state["tokens"].shape
    loss = torch.zeros(case["N"], dtype=torch.float64, device="cuda")
    norm = torch.zeros_like(loss)
    gx, gw = torch.zeros_like(x), torch.zeros_like(w)
    for at in kept.split(1024):
        z = x[at] @ w.T
        norm[at] = torch.logsumexp(z, 1)
        loss[at] = norm[at] - z[torch.arange(len(at), device="cuda"), tokens[at]]
        if op == "xent_train":
            p = torch.softmax(z, 1)
            p[torch.arange(len(at), device="cuda"), tokens[at]] -= 1.0
            p *= _loss_scale(case) / len(kept)
            gx[at] = p @ w
            gw += p.T @ x[at]
    got = {"loss": loss.view(shape), "lse": norm.view(shape)}
    if op == "xent_train":
        got["gx"], got["gw"] = from_rows(gx), gw
    return got


def work(case):
    b = BYTES[case["type"]]
    if case["op"] == "grad_norm":
        return {"bytes": case["total"] * b, "flops": 2 * case["total"]}
    if case["op"] == "grad_clip":
        return {"bytes": 2 * case["total"] * b, "flops": 3 * case["total"]}
    N, D, V = case["N"], case["D"], case["V"]
    live = max(1, int(N * case["kept"]))
    if case["op"] == "embedding_fprop":
        # rows met several times are read once
        return {"bytes": min(live, V) * D * b + N * D * b + N * 8, "flops": N * D}
    if case["op"] == "embedding_accgrad":
        return {"bytes": live * D * b + V * D * b + N * 8, "flops": live * D}
    bytes_ = live * D * b + V * D * b + N * 16
    if case["op"] == "xent_fprop":
        return {"bytes": bytes_, "flops": 2 * live * D * V}
    return {"bytes": bytes_ + N * D * b + V * D * b, "flops": 6 * live * D * V}
