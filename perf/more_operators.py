"""Measured cases of a token model's two ends and of the bound on its step.

Three operators, each in a plain form (elementary torch operations in 32 bits, 64 where sums are long)
and through the library's public entry points:

  lookup  out_i = s E[t_i], a row of zeros where t_i is no row of E;  dE_v = s sum of dout_i over t_i = v
  loss    z = s h W^T, loss_i = log sum_j exp z_ij - z_{i,t_i}, total = sum_i g_i loss_i with
          g_i = 1 / (rows that have a target), 0 for the others;  dh and dW of total
  clip    norm = sqrt(sum of squares over all tensors), each tensor times min(1, most / norm)

"grad" cases run the forward and the backward pass, as a training step does.
"""
import math

import torch

own = False

MOST = 1.0            # bound of the gradient's norm


# ---- cases ------------------------------------------------------------------------------------

def listed():
    return [
        # serving: the next token of each of 16 sequences
        {"name": "lookup 16 of 32768x2048", "op": "lookup", "N": 16, "V": 32768, "D": 2048, "dtype": "bf16",
         "grad": False, "ids": "i64", "common": 0.0},
        # a training step over 16384 tokens, and the gradient of the whole table
        {"name": "lookup grad 16384 of 32768x2048", "op": "lookup", "N": 16384, "V": 32768, "D": 2048, "dtype": "bf16",
         "grad": True, "ids": "i64", "common": 0.0},
        # odd sizes in fp32; half of the batch is one and the same padding token
        {"name": "lookup grad 5003 of 10007x515", "op": "lookup", "N": 5003, "V": 10007, "D": 515, "dtype": "f32",
         "grad": True, "ids": "i32", "common": 0.5},
        # serving: how likely were 16 sampled tokens
        {"name": "loss 16x32768x2048", "op": "loss", "N": 16, "V": 32768, "D": 2048, "dtype": "bf16", "grad": False,
         "left_out": 0.0},
        # evaluation over a batch of prompts
        {"name": "loss 8192x32768x2048", "op": "loss", "N": 8192, "V": 32768, "D": 2048, "dtype": "bf16",
         "grad": False, "left_out": 0.0},
        # a training step
        {"name": "loss grad 8192x32768x2048", "op": "loss", "N": 8192, "V": 32768, "D": 2048, "dtype": "bf16",
         "grad": True, "left_out": 0.0},
        # odd sizes in fp32; four rows in ten are prompts or padding without a target
        {"name": "loss grad 1003x5003x515 ragged", "op": "loss", "N": 1003, "V": 5003, "D": 515, "dtype": "f32",
         "grad": True, "left_out": 0.4},
        # a training step in fp32
        {"name": "loss grad 2048x32768x1024", "op": "loss", "N": 2048, "V": 32768, "D": 1024, "dtype": "f32",
         "grad": True, "left_out": 0.0},
        # a large vocabulary and wide rows
        {"name": "loss grad 4096x131072x4096", "op": "loss", "N": 4096, "V": 131072, "D": 4096, "dtype": "bf16",
         "grad": True, "left_out": 0.1},
        # the gradients of a small stack: latency counts
        {"name": "clip 16 small", "op": "clip", "shapes": "64x64,64", "count": 8, "dtype": "f32", "size": 0.05},
        # every weight of a deep net: 64 layers of width 1024
        {"name": "clip 64 of 1024x1024", "op": "clip", "shapes": "1024x1024", "count": 64, "dtype": "f32",
         "size": 0.05},
        # bf16 gradients of odd sizes
        {"name": "clip 96 odd", "op": "clip", "shapes": "1537x677,677,2048x511", "count": 32, "dtype": "bf16",
         "size": 0.02},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    d = _log(rng, lo, hi)
    return max(64, d // 64 * 64) if rng.random() < 0.6 else d


def draw(rng):
    op = rng.choice(["lookup", "loss", "loss", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "lookup":
        D, V = _width(rng, 16, 4096), _log(rng, 64, 131072)
        V = max(64, min(V, (1 << 27) // D))
        return {"op": "lookup", "N": _log(rng, 1, max(1, min(65536, (1 << 26) // D))), "V": V, "D": D, "dtype": dtype,
                "grad": rng.random() < 0.6, "ids": rng.choice(["i64", "i32"]), "common": rng.choice([0.0, 0.0, 0.3])}
    if op == "loss":
        D, V = _width(rng, 64, 4096), _log(rng, 64, 131072)
        V = max(64, min(V, (1 << 28) // D))
        most = (1 << 37) if dtype == "bf16" else (1 << 36)
        return {"op": "loss", "N": _log(rng, 1, max(1, min(16384, most // (V * D)))), "V": V, "D": D, "dtype": dtype,
                "grad": rng.random() < 0.6, "left_out": rng.choice([0.0, 0.0, 0.3])}
    shapes, size = [], 0
    for _ in range(rng.randint(1, 4)):
        a, b = _log(rng, 1, 4096), _log(rng, 1, 4096)
        shapes.append(f"{a}x{b}")
        size += a * b
    return {"op": "clip", "shapes": ",".join(shapes), "count": _log(rng, 1, max(1, min(64, (1 << 26) // size))),
            "dtype": dtype, "size": rng.choice([0.05, 1e-5])}


def _sizes(c):
    return [tuple(int(n) for n in s.split("x")) for s in c["shapes"].split(",")] * c["count"]


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "lookup":
        n, t = c["N"] * c["D"], c["N"] * (8 if c["ids"] == "i64" else 4)
        if c["grad"]:        # rows read and written; then dout read and the table's gradient written
            return {"bytes": 3 * e * n + e * c["V"] * c["D"] + 2 * t, "flops": 2 * n}
        return {"bytes": 2 * e * n + t, "flops": n}
    if c["op"] == "loss":
        live = max(1, round(c["N"] * (1 - c["left_out"])))
        p, ends = 2.0 * live * c["V"] * c["D"], e * (c["N"] + c["V"]) * c["D"] + 12 * c["N"]
        if c["grad"]:        # the logits, dh and dW
            return {"bytes": 2 * ends, "flops": 3 * p}
        return {"bytes": ends, "flops": p}
    n = sum(math.prod(s) for s in _sizes(c))
    return {"bytes": 2 * e * n, "flops": 3 * n}


# ---- inputs -----------------------------------------------------------------------------------

def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _bucket(tensors, dtype):
    """(an array of zeros, a window of it for each tensor); windows start on multiples of 128 elements."""
    at, n = [], 0
    for t in tensors:
        at.append(n)
        n += -(-t.numel() // 128) * 128
    bucket = torch.zeros(n, device="cuda", dtype=dtype)
    return bucket, [bucket[i:i + t.numel()].view(t.shape) for i, t in zip(at, tensors)]


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = _dtype(c)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dt).mul_(std)

    def uniform(n):
        return torch.rand(n, generator=g, device="cuda")

    def tokens(n, V):
        # frequencies fall as 1 / rank, and ranks are spread over the ids
        rank = (torch.exp(uniform(n) * math.log(V)) - 1).long().clamp_(0, V - 1)
        return torch.randperm(V, generator=g, device="cuda")[rank]

    s = {"case": c}
    if c["op"] == "lookup":
        N, V, D = c["N"], c["V"], c["D"]
        s["table"] = normal(V, D, std=0.02)
        t = tokens(N, V)
        if c["common"]:
            t = torch.where(uniform(N) < c["common"], V // 2, t)
        s["tokens"] = t.to(torch.int64 if c["ids"] == "i64" else torch.int32)
        s["scale"] = math.sqrt(D)
        if c["grad"]:
            s["dout"] = normal(N, D)
    elif c["op"] == "loss":
        N, V, D = c["N"], c["V"], c["D"]
        s["W"] = normal(V, D, std=1.0 / math.sqrt(D))
        t = tokens(N, V)
        # normed states that lean towards their targets: some rows are sure, some know nothing
        s["h"] = normal(N, D).add_(s["W"][t] * (12.0 * uniform(N)[:, None]).to(dt))
        if c["left_out"]:
            out = uniform(N) < c["left_out"]
            t = torch.where(out, -100, t)
            s["h"][out] = float("nan")          # what stands there must not matter
        s["targets"] = t
        s["scale"] = 1.0
    else:
        s["grads"] = [normal(*shape, std=c["size"]) for shape in _sizes(c)]
        # the clipped gradients go into one array, where a data-parallel step would reduce them
        s["bucket"], s["out"] = _bucket(s["grads"], dt)
    return s


# ---- plain forms ------------------------------------------------------------------------------

def _plain_lookup(s):
    c, dt, t = s["case"], _dtype(s["case"]), s["tokens"].long()
    ok = (t >= 0) & (t < c["V"])
    rows = s["table"][torch.where(ok, t, 0)].float() * s["scale"]
    out = {"out": torch.where(ok[:, None], rows, 0.0).to(dt)}
    if c["grad"]:
        d = torch.where(ok[:, None], s["dout"].float() * s["scale"], 0.0)
        sums = torch.zeros(c["V"], c["D"], device=t.device)
        out["dtable"] = sums.index_add_(0, torch.where(ok, t, 0), d).to(dt)
    return out


def _plain_loss(s):
    c, dt, t = s["case"], _dtype(s["case"]), s["targets"]
    N, V = c["N"], c["V"]
    W = s["W"].float()
    live = (t >= 0) & (t < V)
    weight = live.float() / live.sum().clamp(min=1)
    loss = torch.zeros(N, device=t.device)
    dh = torch.zeros(N, c["D"], device=t.device, dtype=dt) if c["grad"] else None
    dW = torch.zeros_like(W) if c["grad"] else None
    for i in range(0, N, 1024):
        on = live[i:i + 1024, None]
        h = torch.where(on, s["h"][i:i + 1024].float(), 0.0)
        z = s["scale"] * (h @ W.T)
        z = z - z.max(1, keepdim=True).values
        e = torch.exp(z)
        total = e.sum(1, keepdim=True)
        at = torch.where(on, t[i:i + 1024, None], 0)
        loss[i:i + 1024] = torch.where(on, torch.log(total) - z.gather(1, at), 0.0)[:, 0]
        if c["grad"]:
            w = s["scale"] * weight[i:i + 1024, None]
            e = e * (w / total)
            e.scatter_add_(1, at, -w)
            dh[i:i + 1024] = (e @ W).to(dt)
            dW += e.T @ h
    out = {"loss": loss, "total": (loss.double() * weight.double()).sum().float()}
    if c["grad"]:
        out.update(dh=dh, dW=dW.to(dt))
    return out


def _plain_clip(s):
    norm = torch.sqrt(sum((t.double() * t.double()).sum() for t in s["grads"]))
    k = torch.where(norm > MOST, MOST / norm, 1.0).float()
    for t, o in zip(s["grads"], s["out"]):
        o.copy_(t.float() * k)
    return {"norm": norm.float(), "grads": s["bucket"]}


# ---- the library's calls ------------------------------------------------------------------------

def _own_lookup(s):
    from paper_2402_14212_b200 import binding as mwb
    out = {"out": mwb.embedding(s["tokens"], s["table"], scale=s["scale"])}
    if s["case"]["grad"]:
        out["dtable"] = mwb.embedding_backward(s["tokens"], s["dout"], s["case"]["V"], scale=s["scale"])
    return out


def _own_loss(s):
    from paper_2402_14212_b200 import binding as mwb
    if not s["case"]["grad"]:
        r = mwb.token_loss(s["h"], s["W"], s["targets"], scale=s["scale"])
        return {"loss": r.loss, "total": r.total}
    r = mwb.token_loss_gradient(s["h"], s["W"], s["targets"], scale=s["scale"])
    return {"loss": r.loss, "total": r.total, "dh": r.dh, "dW": r.dweight}


def _own_clip(s):
    from paper_2402_14212_b200 import binding as mwb
    return {"norm": mwb.clip_gradients(s["grads"], MOST, out=s["out"]), "grads": s["bucket"]}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"lookup": _own_lookup, "loss": _own_loss, "clip": _own_clip}[op](s)
    return {"lookup": _plain_lookup, "loss": _plain_loss, "clip": _plain_clip}[op](s)


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    return {"lookup": _exact_lookup, "loss": _exact_loss, "clip": _exact_clip}[c["op"]](s)


def _exact_lookup(s):
    """Rows by their ids; the gradient by automatic differentiation."""
    c, t = s["case"], s["tokens"].long()
    out = {"out": torch.nn.functional.embedding(t, s["table"].double()) * s["scale"]}
    if c["grad"]:
        leaf = torch.zeros(c["V"], c["D"], device=t.device, dtype=torch.float64, requires_grad=True)
        y = torch.nn.functional.embedding(t, leaf) * s["scale"]
        out["dtable"], = torch.autograd.grad(y, leaf, s["dout"].double())
    return out


def _exact_loss(s):
    """Forward from the definition, a few rows at a time; gradients by automatic differentiation."""
    c = s["case"]
    keep = ((s["targets"] >= 0) & (s["targets"] < c["V"])).nonzero()[:, 0]
    W = s["W"].double().requires_grad_(c["grad"])
    loss = torch.zeros(c["N"], device=W.device, dtype=torch.float64)
    dh = torch.zeros(c["N"], c["D"], device=W.device, dtype=torch.float64)
    total = torch.zeros((), device=W.device, dtype=torch.float64)
    step = max(1, (1 << 27) // c["V"])
    for rows in keep.split(step):
        h = s["h"][rows].double().requires_grad_(c["grad"])
        part = torch.nn.functional.cross_entropy(s["scale"] * (h @ W.T), s["targets"][rows], reduction="none")
        loss[rows] = part.detach()
        part = part.sum() / len(keep)
        total += part.detach()
        if c["grad"]:
            part.backward()
            dh[rows] = h.grad
    out = {"loss": loss, "total": total}
    if c["grad"]:
        out.update(dh=dh, dW=torch.zeros_like(W) if W.grad is None else W.grad)
    return out


def _exact_clip(s):
    """The norm of the tensors' norms."""
    g = [t.double() for t in s["grads"]]
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t) for t in g]))
    k = MOST / max(MOST, float(norm))
    bucket, out = _bucket(g, torch.float64)
    for t, o in zip(g, out):
        torch.mul(t, k, out=o)
    return {"norm": norm, "grads": bucket}
