"""What the operators at both ends of a model over a vocabulary cost: embedding lookup and its gradient, layer norm and its
backprop, and softmax cross entropy of a linear layer with the gradients of both its operands.

listed() names twelve cases, draw() gives further ones of the same ranges; prepare() builds what a user's program holds before
the calls and run() makes one pass.  With `own` set it makes the calls of the package; otherwise it computes the same results
from elementary torch operations in 32 bits, rounded once at the end.  A case is a dict of plain values:

  op      "embedding" | "embedding_bwd" | "norm" | "norm_bwd" | "xent" | "xent_step" (loss, then both gradients)
  dtype   element type of the data tensors: "bf16" | "f32"
  rows    tokens
  width   elements of a token's row
  vocab   rows of the table or of the linear layer's weight (not for norms)
"""
import math

import torch

own = False

EPS = 1e-5
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(op, dtype, rows, width, vocab=0):
    return {"op": op, "dtype": dtype, "rows": rows, "width": width, "vocab": vocab}


def listed():
    return [
        # One decode step of eight sequences: the rows of eight tokens.  Latency only.
        dict(_case("embedding", "bf16", 8, 2048, 32000), name="embed_decode"),
        # The input of a training step: 32768 tokens over a vocabulary of no round size.
        dict(_case("embedding", "bf16", 32768, 4096, 50257), name="embed_batch"),
        # Its gradient on a smaller model: frequent tokens have hundreds of positions, most of the vocabulary none.
        dict(_case("embedding_bwd", "bf16", 16384, 2048, 32000), name="embed_grad"),
        # Full precision, nothing a multiple of anything.
        dict(_case("embedding_bwd", "f32", 5001, 777, 10007), name="embed_grad_odd"),
        # The norm in front of a decode step's layers.  Latency only.
        dict(_case("norm", "bf16", 8, 4096), name="norm_decode"),
        # The norm of a training step's tokens, and its backprop.
        dict(_case("norm", "bf16", 16384, 4096), name="norm_batch"),
        dict(_case("norm_bwd", "bf16", 16384, 4096), name="norm_grad"),
        dict(_case("norm_bwd", "f32", 3001, 1001), name="norm_grad_odd"),
        # Scoring text: the loss alone, no gradients.
        dict(_case("xent", "bf16", 2048, 2048, 32000), name="xent_eval"),
        # The loss of a training step with the gradients of the activations and the weight.  The largest case.
        dict(_case("xent_step", "bf16", 8192, 4096, 50257), name="xent_step"),
        # The classifier behind an image network: 2048 features, 1000 classes, a batch of 128.
        dict(_case("xent_step", "bf16", 128, 2048, 1000), name="xent_head"),
        # Full precision, nothing a multiple of anything.
        dict(_case("xent_step", "f32", 1000, 515, 10007), name="xent_step_odd"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(("embedding", "embedding_bwd", "norm", "norm_bwd", "xent", "xent_step", "xent_step"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    while True:
        rows = _log(rng, 1, 65536 if op.startswith("embedding") else 32768 if op.startswith("norm") else 8192)
        width = _log(rng, 16, 16384 if op.startswith("norm") else 4096)
        if rng.random() < 0.5:
            width = max(64, width // 64 * 64)            # model widths are usually round; the other half is anything
        vocab = 0 if op.startswith("norm") else _log(rng, 100, 65536)
        case = _case(op, dtype, rows, width, vocab)
        if op.startswith("xent"):
            fits = rows * width * vocab <= (1 << 37 if dtype == "f32" else 1 << 40)
        else:
            fits = rows * width <= 1 << 27 and vocab * width <= 1 << 28
        if fits:
            return case


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, rows, width, vocab = _TYPES[case["dtype"]], case["rows"], case["width"], case["vocab"]
    normal = lambda shape, std: torch.randn(shape, generator=gen, device="cuda") * std
    state = {"case": case}
    if vocab:
        # Tokens as text has them: the frequency falls with the rank.  The last twentieth is padding, which has no row.
        u = torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * math.log(vocab)) - 1).long().clamp_(0, vocab - 1)
        ids[rows - rows // 20:] = -1
        state["ids"] = ids
    if case["op"].startswith("embedding"):
        state["scale"] = float(width) ** 0.5
        if case["op"] == "embedding":
            state["table"] = normal((vocab, width), 0.02).to(dtype)
        else:
            state["dy"] = normal((rows, width), 1e-3).to(dtype)
    elif case["op"].startswith("norm"):
        # A residual stream: some features far from zero, row scales that differ.
        offset = normal((width,), 1.0) * (torch.rand(width, generator=gen, device="cuda") < 0.02) * 20
        x = normal((rows, width), 1.0) * (0.5 + torch.rand((rows, 1), generator=gen, device="cuda")) + offset
        state["x"] = x.to(dtype)
        state["gamma"] = 1 + normal((width,), 0.1)
        state["beta"] = normal((width,), 0.1)
        if case["op"] == "norm_bwd":
            state["dy"] = normal((rows, width), 1e-3).to(dtype)
            x = state["x"].double()                      # what the forward pass left
            mean = x.mean(1)
            state["mean"], state["rstd"] = mean.float(), (((x - mean[:, None]) ** 2).mean(1) + EPS).rsqrt().float()
    else:
        w = normal((vocab, width), 0.02)
        # Activations of a model that has learnt something: the label's logit stands out from the others by up to six.
        lift = torch.rand((rows, 1), generator=gen, device="cuda") * 6 / (0.02 * 0.02 * width)
        state["x"] = (normal((rows, width), 1.0) + lift * w[state["ids"].clamp_min(0)]).to(dtype)
        state["w"] = w.to(dtype)
        # The mean over the rows that count.
        state["dloss"] = torch.full((rows,), 1.0 / max(1, rows - rows // 20), device="cuda")
    return state


# --------------------------------------------------------------------------------------------------- plain forms

def _plain_embedding(state):
    ids, table = state["ids"], state["table"]
    live = (ids >= 0) & (ids < table.shape[0])
    y = table[ids.clamp(0, table.shape[0] - 1)].float() * state["scale"]
    return {"y": torch.where(live[:, None], y, 0.0).to(table.dtype)}


def _plain_embedding_bwd(state):
    ids, dy, vocab = state["ids"], state["dy"], state["case"]["vocab"]
    live = (ids >= 0) & (ids < vocab)
    dtable = torch.zeros((vocab, dy.shape[1]), device="cuda")
    dtable.index_add_(0, ids.clamp(0, vocab - 1), torch.where(live[:, None], dy.float(), 0.0))
    return {"dtable": dtable * state["scale"]}


def _plain_norm(state):
    x = state["x"].float()
    mean = x.mean(1, keepdim=True)
    rstd = torch.rsqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    y = (x - mean) * rstd * state["gamma"] + state["beta"]
    return {"y": y.to(state["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}


def _plain_norm_bwd(state):
    dy, rstd = state["dy"].float(), state["rstd"][:, None]
    xhat = (state["x"].float() - state["mean"][:, None]) * rstd
    g = dy * state["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return {"dx": dx.to(state["x"].dtype), "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}


def _plain_xent(state, grads):
    x, w, labels = state["x"].float(), state["w"].float(), state["ids"]
    live = (labels >= 0) & (labels < w.shape[0])
    at = labels.clamp(0, w.shape[0] - 1)[:, None]
    logits = x @ w.T
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    got = {"loss": torch.where(live, lse - logits.gather(1, at)[:, 0], 0.0), "lse": lse}
    if grads:
        g = e / total
        g.scatter_add_(1, at, torch.full_like(total, -1.0))
        g = g * torch.where(live, state["dloss"], 0.0)[:, None]
        got["dx"], got["dw"] = (g @ w).to(state["x"].dtype), (g.T @ x).to(state["w"].dtype)
    return got


# --------------------------------------------------------------------------------------------------- the package's calls

def _buffers(state):
    """Outputs and workspaces, allocated once: a user's program keeps them from step to step."""
    if "out" not in state:
        import paper_1801_08058_amd as ng
        case = state["case"]
        code = ng.NGC_F32 if case["dtype"] == "f32" else ng.NGC_BF16
        rows, width, vocab, op = case["rows"], case["width"], case["vocab"], case["op"]
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")
        data = _TYPES[case["dtype"]]
        need = 0
        if op == "embedding":
            out = {"y": new(rows, width, dtype=data)}
        elif op == "embedding_bwd":
            out = {"dtable": new(vocab, width)}
            need = ng.ngc_embedding_workspace_bytes(rows, vocab, width)
        elif op == "norm":
            out = {"y": new(rows, width, dtype=data), "mean": new(rows), "rstd": new(rows)}
        elif op == "norm_bwd":
            out = {"dx": new(rows, width, dtype=data), "dgamma": new(width), "dbeta": new(width)}
            need = ng.ngc_layer_norm_workspace_bytes(code, rows, width)
        else:
            out = {"loss": new(rows), "lse": new(rows)}
            need = ng.ngc_linear_xent_workspace_bytes(code, rows, width, vocab, 0)
            if op == "xent_step":
                out["dx"], out["dw"] = new(rows, width, dtype=data), new(vocab, width, dtype=data)
                need = max(need, ng.ngc_linear_xent_workspace_bytes(code, rows, width, vocab, 1))
        state["ng"], state["code"], state["out"] = ng, code, out
        state["ws"] = new(need, dtype=torch.uint8) if need else None
    return state["ng"], state["code"], state["out"], state["ws"]


def _own(state):
    ng, code, out, ws = _buffers(state)
    case, stream = state["case"], torch.cuda.current_stream().cuda_stream
    rows, width, vocab, op = case["rows"], case["width"], case["vocab"], case["op"]
    if op == "embedding":
        ng.ngc_embedding(code, rows, vocab, width, state["scale"], state["table"], state["ids"], out["y"], stream)
    elif op == "embedding_bwd":
        ng.ngc_embedding_bwd(code, rows, vocab, width, state["scale"], state["dy"], state["ids"], out["dtable"], ws, stream)
    elif op == "norm":
        ng.ngc_layer_norm(code, rows, width, EPS, state["x"], state["gamma"], state["beta"], out["y"], out["mean"], out["rstd"], stream)
    elif op == "norm_bwd":
        ng.ngc_layer_norm_bwd(code, rows, width, state["x"], state["gamma"], state["mean"], state["rstd"], state["dy"], out["dx"],
                              out["dgamma"], out["dbeta"], ws, stream)
    else:
        ng.ngc_linear_xent(code, rows, width, vocab, state["x"], state["w"], state["ids"], out["loss"], out["lse"], ws, stream)
        if op == "xent_step":
            ng.ngc_linear_xent_bwd(code, rows, width, vocab, state["x"], state["w"], state["ids"], out["lse"], state["dloss"], out["dx"],
                                   out["dw"], ws, stream)
    return out


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op.startswith("xent"):
        return _plain_xent(state, op == "xent_step")
    return {"embedding": _plain_embedding, "embedding_bwd": _plain_embedding_bwd, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd}[op](state)


# --------------------------------------------------------------------------------------------------- accounting and exact values

def work(case):
    rows, width, vocab, op = case["rows"], case["width"], case["vocab"], case["op"]
    size = 4 if case["dtype"] == "f32" else 2
    data = rows * width * size
    if op == "embedding":
        return {"bytes": 2 * data + 8 * rows, "flops": rows * width}
    if op == "embedding_bwd":
        return {"bytes": data + 8 * rows + 4 * vocab * width, "flops": 2 * rows * width}
    if op == "norm":
        return {"bytes": 2 * data + 8 * width + 8 * rows, "flops": 8 * rows * width}
    if op == "norm_bwd":
        return {"bytes": 3 * data + 12 * width + 8 * rows, "flops": 14 * rows * width}
    weight, product = vocab * width * size, 2 * rows * width * vocab
    if op == "xent":
        return {"bytes": data + weight + 16 * rows, "flops": product}
    return {"bytes": 2 * data + 2 * weight + 20 * rows, "flops": 3 * product}


def exact(case, seed):
    state = prepare(case, seed)
    op, vocab = case["op"], case["vocab"]
    if op == "embedding":
        padded = torch.cat([state["table"].double() * state["scale"], torch.zeros((1, case["width"]), dtype=torch.float64, device="cuda")])
        return {"y": padded[torch.where((state["ids"] < 0) | (state["ids"] >= vocab), vocab, state["ids"])]}
    if op == "embedding_bwd":
        spare = torch.zeros((vocab + 1, case["width"]), dtype=torch.float64, device="cuda")
        rows = torch.where((state["ids"] < 0) | (state["ids"] >= vocab), vocab, state["ids"])
        return {"dtable": spare.index_add_(0, rows, state["dy"].double() * state["scale"])[:vocab]}
    if op == "norm":
        x = state["x"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        std = torch.sqrt(var + EPS)
        return {"y": (x - mean[:, None]) / std[:, None] * state["gamma"].double() + state["beta"].double(), "mean": mean, "rstd": 1 / std}
    if op == "norm_bwd":
        # Of the forward pass from the statistics that were handed over, not from those of x.
        x, dy, gamma = state["x"].double(), state["dy"].double(), state["gamma"].double()
        rstd = state["rstd"].double()[:, None]
        centred = x - state["mean"].double()[:, None]
        along = (dy * gamma * centred).sum(1, keepdim=True) * rstd ** 2 / case["width"]
        dx = rstd * (dy * gamma - (dy * gamma).sum(1, keepdim=True) / case["width"] - centred * along)
        return {"dx": dx, "dgamma": (dy * (centred * rstd)).sum(0), "dbeta": dy.sum(0)}
    x, w, labels = state["x"].double(), state["w"].double(), state["ids"]
    dead = (labels < 0) | (labels >= vocab)
    at = torch.where(dead, 0, labels)
    z = torch.mm(x, w.t().contiguous())
    lse = torch.logsumexp(z, 1)
    got = {"loss": (lse - z[torch.arange(case["rows"], device="cuda"), at]).masked_fill(dead, 0.0), "lse": lse}
    if op == "xent_step":
        z.sub_(lse[:, None]).exp_()
        z[torch.arange(case["rows"], device="cuda"), at] -= 1
        z.mul_(state["dloss"].double().masked_fill(dead, 0.0)[:, None])
        got["dx"], got["dw"] = torch.mm(z, w), torch.mm(z.t().contiguous(), x)
    return got
