"""Measured cases of the sequence-block operators and the orthogonalised update.

Three operators, each in a plain form (elementary torch operations in 32 bits) and through the
library's public entry points:

  scan    gated linear recurrence  h_t = r_t a_t h_{t-1} + u_t v_t,  a = sigmoid(f),
          u = 1 - a ("complement") or sqrt(1 - a^2) ("energy"), r_t = 0 at a reset
  norm    x' = x + s silu(z) rmsnorm(b; w_post),  n = rmsnorm(x'; w_pre)
  orth    orthogonalised momentum update: five quintic Newton-Schulz steps on the (Nesterov)
          momentum, then W' = (1 - lr wd) W - lr s X; or the projection X alone

"grad" cases run the forward and the backward pass, as a training step does.
"""
import math

import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-6
BETA, LR, DECAY = 0.95, 0.02, 0.01


# ---- cases ------------------------------------------------------------------------------------

def listed():
    return [
        # serving: one token for each of 64 sequences, recurrent state carried in
        {"name": "scan token 64x1x2048", "op": "scan", "B": 64, "T": 1, "D": 2048, "dtype": "bf16",
         "gate": "complement", "grad": False, "ragged": False},
        # prefill of a batch of prompts
        {"name": "scan 8x2048x2048", "op": "scan", "B": 8, "T": 2048, "D": 2048, "dtype": "bf16",
         "gate": "complement", "grad": False, "ragged": False},
        # one very long sequence: few channels, the time axis has to be split
        {"name": "scan 1x65536x1024", "op": "scan", "B": 1, "T": 65536, "D": 1024, "dtype": "bf16",
         "gate": "energy", "grad": False, "ragged": False},
        # a training step's forward and backward pass
        {"name": "scan grad 4x4096x2048", "op": "scan", "B": 4, "T": 4096, "D": 2048, "dtype": "bf16",
         "gate": "complement", "grad": True, "ragged": False},
        # packed and padded sequences of odd sizes in fp32, one of them empty
        {"name": "scan grad 5x1003x515 ragged", "op": "scan", "B": 5, "T": 1003, "D": 515, "dtype": "f32",
         "gate": "energy", "grad": True, "ragged": True},
        # serving: the residual step of 16 tokens
        {"name": "norm 16x2048", "op": "norm", "R": 16, "D": 2048, "dtype": "bf16", "grad": False},
        # a training step over 16384 tokens
        {"name": "norm grad 16384x4096", "op": "norm", "R": 16384, "D": 4096, "dtype": "bf16", "grad": True},
        # odd sizes in fp32
        {"name": "norm grad 1003x1111", "op": "norm", "R": 1003, "D": 1111, "dtype": "f32", "grad": True},
        # four small weights: latency counts
        {"name": "orth 4 of 64x64", "op": "orth", "L": 4, "rows": 64, "cols": 64, "dtype": "f32", "step": True},
        # every weight of a deep MLP: 64 layers of width 1024 in fp32
        {"name": "orth 64 of 1024x1024", "op": "orth", "L": 64, "rows": 1024, "cols": 1024, "dtype": "f32",
         "step": True},
        # wide layers with bf16 weights
        {"name": "orth 2 of 4096x4096", "op": "orth", "L": 2, "rows": 4096, "cols": 4096, "dtype": "bf16",
         "step": True},
        # projection of tall matrices of odd sizes
        {"name": "orth project 3 of 1537x677", "op": "orth", "L": 3, "rows": 1537, "cols": 677, "dtype": "bf16",
         "step": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["scan", "scan", "norm", "orth"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "scan":
        grad = rng.random() < 0.5
        B, D = _log(rng, 1, 64), _log(rng, 64, 4096)
        if rng.random() < 0.6:
            D = max(64, D // 64 * 64)
        most = (1 << 25) if grad else (1 << 26)
        T = 1 if (not grad and rng.random() < 0.25) else _log(rng, 2, max(2, min(65536, most // (B * D))))
        return {"op": "scan", "B": B, "T": T, "D": D, "dtype": dtype, "gate": rng.choice(["complement", "energy"]),
                "grad": grad, "ragged": rng.random() < 0.4}
    if op == "norm":
        D = _log(rng, 64, 8192)
        if rng.random() < 0.6:
            D = max(64, D // 64 * 64)
        return {"op": "norm", "R": _log(rng, 1, max(1, min(65536, (1 << 26) // D))), "D": D, "dtype": dtype,
                "grad": rng.random() < 0.6}
    rows, cols = _log(rng, 33, 4096), _log(rng, 33, 4096)
    if rng.random() < 0.5:
        cols = rows
    m, n = min(rows, cols), max(rows, cols)
    most = (1.4e11 if dtype == "bf16" else 6.8e10) / (3.0 * m * m * n + float(m) ** 3) * 4
    L = _log(rng, 1, max(1, min(64, int(most))))
    return {"op": "orth", "L": L, "rows": rows, "cols": cols, "dtype": dtype, "step": rng.random() < 0.7}


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "scan":
        n = c["B"] * c["T"] * c["D"]
        state = 4 * c["B"] * c["D"]
        if c["grad"]:        # v, f read and y written; then v, f, dy read and dv, df written
            return {"bytes": 8 * e * n + 5 * state, "flops": 40 * n}
        return {"bytes": 3 * e * n + 2 * state, "flops": 14 * n}
    if c["op"] == "norm":
        n = c["R"] * c["D"]
        if c["grad"]:        # x, b, z read, x', n written; then x, b, z, dx', dn read, dx, db, dz written
            return {"bytes": 13 * e * n + 24 * c["D"], "flops": 60 * n}
        return {"bytes": 5 * e * n + 12 * c["D"], "flops": 20 * n}
    m, n = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    k = c["L"] * m * n
    # two symmetric products (half each) and one full one per step
    flops = 5.0 * c["L"] * (3.0 * m * m * n + float(m) ** 3)
    return {"bytes": (12 * k + 2 * e * k) if c["step"] else 2 * e * k, "flops": flops}


# ---- inputs -----------------------------------------------------------------------------------

def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = _dtype(c)

    def normal(*shape, mean=0.0, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)

    s = {"case": c}
    if c["op"] == "scan":
        B, T, D = c["B"], c["T"], c["D"]
        # one projection yields values and decay logits side by side: both are windows of its rows.
        # Channels remember over a few to a few hundred steps.
        vf = torch.empty(B, T, 2 * D, device="cuda", dtype=dt)
        vf[:, :, :D] = normal(B, T, D)
        vf[:, :, D:] = (torch.randn(B, T, D, generator=g, device="cuda") +
                        torch.linspace(0.0, 5.0, D, device="cuda")).to(dt)
        s["v"], s["f"] = vf[:, :, :D], vf[:, :, D:]
        s["h0"] = normal(B, D, std=0.5, dtype=torch.float32)
        s["reset"] = s["lengths"] = None
        if c["ragged"]:
            s["reset"] = (torch.rand(B, T, generator=g, device="cuda") < 0.01).to(torch.uint8)
            n = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            n[0], n[-1] = T, 0
            s["lengths"] = n
            # what stands in the padding must not matter
            past = torch.arange(T, device="cuda")[None, :] >= n[:, None]
            vf[past] = float("nan")
        if c["grad"]:
            s["dy"] = normal(B, T, D)
            s["dh_last"] = normal(B, D, dtype=torch.float32)
    elif c["op"] == "norm":
        R, D = c["R"], c["D"]
        s["x"] = normal(R, D, std=2.0)
        s["b"], s["z"] = normal(R, D, std=0.7), normal(R, D)
        s["w_post"], s["w_pre"] = (normal(D, mean=1.0, std=0.1, dtype=torch.float32) for _ in range(2))
        s["scale"] = normal(D, mean=0.3, std=0.05, dtype=torch.float32)
        if c["grad"]:
            s["dx_out"], s["dn"] = normal(R, D), normal(R, D)
    else:
        L, m, n = c["L"], c["rows"], c["cols"]
        # gradients of a batch: a few strong directions over a broad floor
        k = max(1, min(m, n) // 8)
        grad = torch.randn(L, m, k, generator=g, device="cuda") @ torch.randn(L, k, n, generator=g, device="cuda")
        grad = grad / math.sqrt(k) + torch.randn(L, m, n, generator=g, device="cuda")
        if c["step"]:
            s["grad"] = grad
            s["momentum"] = torch.randn(L, m, n, generator=g, device="cuda")
            s["W"] = normal(L, m, n, std=1.0 / math.sqrt(max(m, n)))
            s["W_out"] = torch.empty_like(s["W"])
            s["m_out"] = torch.empty_like(s["momentum"])
            s["scale"] = 0.2 * math.sqrt(max(m, n))
        else:
            s["U"] = grad.to(dt)
            s["X_out"] = torch.empty_like(s["U"])
        if own:
            from paper_2402_14212_b200 import binding as mwb
            s["plan"] = mwb.Orth(m, n, L, "f32" if c["dtype"] == "f32" else "bf16_f32acc")
            s["ws"] = s["plan"].alloc_workspace()
    return s


# ---- plain forms ------------------------------------------------------------------------------

def _shift(x, k, fill):
    """x moved k steps later along dim 1, the first k steps filled."""
    return torch.cat([torch.full_like(x[:, :k], fill), x[:, :-k]], 1)


def _linear_scan(A, b):
    """h_t = A_t h_{t-1} + b_t over dim 1 from h = 0, by doubling."""
    k = 1
    while k < b.shape[1]:
        b = b + A * _shift(b, k, 0.0)
        A = A * _shift(A, k, 1.0)
        k *= 2
    return b


def _scan_parts(s):
    c = s["case"]
    v, f = s["v"].float(), s["f"].float()
    live = None
    if s["lengths"] is not None:
        live = (torch.arange(c["T"], device=v.device)[None, :] < s["lengths"][:, None])[:, :, None]
        v, f = torch.where(live, v, 0.0), torch.where(live, f, 0.0)
    a, w = 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(f))        # a and 1 - a
    u = w if c["gate"] == "complement" else torch.sqrt(w * (1 + a))
    du = torch.full_like(a, -1.0) if c["gate"] == "complement" else -a / u
    keep = a if s["reset"] is None else a * (1 - s["reset"].float())[:, :, None]
    if live is not None:      # beyond the end the state is held and nothing is added
        keep, u = torch.where(live, keep, 1.0), torch.where(live, u, 0.0)
    return v, a, w, u, du, keep, live


def _plain_scan(s):
    c = s["case"]
    v, a, w, u, du, keep, live = _scan_parts(s)
    b = u * v
    b[:, 0] = b[:, 0] + keep[:, 0] * s["h0"]
    h = _linear_scan(keep, b)
    y = h if live is None else torch.where(live, h, 0.0)
    out = {"y": y.to(_dtype(c)), "h_last": h[:, -1].clone()}
    if c["grad"]:
        dy = s["dy"].float()
        if live is not None:
            dy = torch.where(live, dy, 0.0)
        dy[:, -1] = dy[:, -1] + s["dh_last"]
        nxt = torch.cat([keep[:, 1:], torch.ones_like(keep[:, :1])], 1)
        g = _linear_scan(nxt.flip(1), dy.flip(1)).flip(1)
        r = 1.0 if s["reset"] is None else (1 - s["reset"].float())[:, :, None]
        before = torch.cat([s["h0"][:, None], h[:, :-1]], 1) * r
        dv, df = u * g, a * w * g * (before + du * v)
        if live is not None:
            dv, df = torch.where(live, dv, 0.0), torch.where(live, df, 0.0)
        out.update(dv=dv.to(_dtype(c)), df=df.to(_dtype(c)), dh0=keep[:, 0] * g[:, 0])
    return out


def _plain_norm(s):
    c, dt = s["case"], _dtype(s["case"])
    x, b, z = s["x"].float(), s["b"].float(), s["z"].float()
    rb = torch.rsqrt((b * b).mean(1, keepdim=True) + EPS)
    bh = b * rb
    sig = 1 / (1 + torch.exp(-z))
    t = s["scale"] * z * sig
    xo = x + t * bh * s["w_post"]
    rx = torch.rsqrt((xo * xo).mean(1, keepdim=True) + EPS)
    xh = xo * rx
    out = {"x_out": xo.to(dt), "n": (xh * s["w_pre"]).to(dt)}
    if c["grad"]:
        dn, dxo = s["dn"].float(), s["dx_out"].float()
        q = dn * s["w_pre"]
        dx = dxo + rx * (q - xh * (q * xh).mean(1, keepdim=True))
        dp = dx * t
        q = dp * s["w_post"]
        db = rb * (q - bh * (q * bh).mean(1, keepdim=True))
        p = bh * s["w_post"]
        dz = dx * s["scale"] * p * sig * (1 + z * (1 - sig))
        out.update(dx=dx.to(dt), db=db.to(dt), dz=dz.to(dt), dw_post=(dp * bh).sum(0),
                   dscale=(dx * z * sig * p).sum(0), dw_pre=(dn * xh).sum(0))
    return out


def _plain_project(U):
    a, b, c = COEF
    X = U / torch.sqrt((U * U).sum((1, 2), keepdim=True))
    tall = X.shape[1] > X.shape[2]
    if tall:
        X = X.transpose(1, 2)
    for _ in range(5):
        A = X @ X.transpose(1, 2)
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.transpose(1, 2) if tall else X


def _plain_orth(s):
    dt = _dtype(s["case"])
    if not s["case"]["step"]:
        return {"X": _plain_project(s["U"].float()).to(dt).contiguous()}
    m = BETA * s["momentum"] + s["grad"]
    X = _plain_project(s["grad"] + BETA * m)
    W = (1 - LR * DECAY) * s["W"].float() - (LR * s["scale"]) * X
    return {"W": W.to(dt), "momentum": m}


# ---- the library's calls ------------------------------------------------------------------------

def _own_scan(s):
    from paper_2402_14212_b200 import binding as mwb
    c = s["case"]
    kw = dict(reset=s["reset"], lengths=s["lengths"], h0=s["h0"], input_gate=c["gate"])
    if not c["grad"]:
        y, h_last = mwb.gated_scan(s["v"], s["f"], **kw)
        return {"y": y, "h_last": h_last}
    y, h_last, kept = mwb.gated_scan(s["v"], s["f"], keep_states=True, **kw)
    dv, df, dh0 = mwb.gated_scan_backward(s["v"], s["f"], s["dy"], kept, dh_last=s["dh_last"], **kw)
    return {"y": y, "h_last": h_last, "dv": dv, "df": df, "dh0": dh0}


def _own_norm(s):
    from paper_2402_14212_b200 import binding as mwb
    kw = dict(z=s["z"], w_post=s["w_post"], scale=s["scale"], w_pre=s["w_pre"], eps=EPS)
    if not s["case"]["grad"]:
        xo, n = mwb.residual_norm(s["x"], s["b"], **kw)
        return {"x_out": xo, "n": n}
    xo, n, rms = mwb.residual_norm(s["x"], s["b"], keep_rms=True, **kw)
    g = mwb.residual_norm_backward(s["x"], s["b"], rms, dx_out=s["dx_out"], dn=s["dn"], **kw)
    return {"x_out": xo, "n": n, "dx": g.dx, "db": g.db, "dz": g.dz, "dw_post": g.dw_post, "dscale": g.dscale,
            "dw_pre": g.dw_pre}


def _own_orth(s):
    if not s["case"]["step"]:
        s["plan"].project(list(s["U"]), s["ws"], out=list(s["X_out"]))
        return {"X": s["X_out"]}
    s["plan"].step(list(s["W"]), list(s["grad"]), list(s["momentum"]), s["ws"], lr=LR, beta=BETA, weight_decay=DECAY,
                   scale=s["scale"], params_out=list(s["W_out"]), momentum_out=list(s["m_out"]))
    return {"W": s["W_out"], "momentum": s["m_out"]}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"scan": _own_scan, "norm": _own_norm, "orth": _own_orth}[op](s)
    return {"scan": _plain_scan, "norm": _plain_norm, "orth": _plain_orth}[op](s)


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(c, seed):
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in prepare(c, seed).items()
         if k not in ("W_out", "m_out", "X_out", "plan", "ws")}
    return {"scan": _exact_scan, "norm": _exact_norm, "orth": _exact_orth}[c["op"]](s)


def _exact_scan(s):
    """Step by step through time."""
    c = s["case"]
    B, T = c["B"], c["T"]
    v, f, h = s["v"], s["f"], s["h0"]
    a = torch.sigmoid(f)
    u = torch.sigmoid(-f)
    if c["gate"] == "energy":
        u = torch.sqrt(u * (1.0 + a))
    r = torch.ones(B, T, 1, device=v.device, dtype=torch.float64)
    if s["reset"] is not None:
        r = 1.0 - s["reset"].double()[:, :, None]
    n = torch.full((B,), T, device=v.device) if s["lengths"] is None else s["lengths"].long()
    hs = torch.empty(B, T, c["D"], device=v.device, dtype=torch.float64)
    ragged = s["lengths"] is not None
    for t in range(T):
        new = torch.addcmul(u[:, t] * v[:, t], r[:, t] * a[:, t], h)
        h = torch.where((t < n)[:, None], new, h) if ragged else new
        hs[:, t] = h
    live = (torch.arange(T, device=v.device)[None, :] < n[:, None])[:, :, None]
    out = {"y": torch.where(live, hs, 0.0), "h_last": h}
    if c["grad"]:
        g = s["dh_last"]
        dv, df = torch.zeros_like(hs), torch.zeros_like(hs)
        for t in range(T - 1, -1, -1):
            on = (t < n)[:, None]
            at, ut, rt = a[:, t], u[:, t], r[:, t]
            gt = g + s["dy"][:, t]
            before = hs[:, t - 1] if t else s["h0"]
            slope = -v[:, t] if c["gate"] == "complement" else -v[:, t] * at / ut
            dv[:, t] = torch.where(on, ut * gt, 0.0)
            df[:, t] = torch.where(on, gt * at * torch.sigmoid(-f[:, t]) * (rt * before + slope), 0.0)
            g = torch.where(on, rt * at * gt, g)
        out.update(dv=dv, df=df, dh0=g)
    return out


def _exact_norm(s):
    """Forward from the definition; gradients by automatic differentiation."""
    names = ("x", "b", "z", "w_post", "scale", "w_pre")
    x, b, z, wp, sc, wn = leaves = [s[k].clone().requires_grad_(s["case"]["grad"]) for k in names]
    xo = x + sc * torch.nn.functional.silu(z) * wp * b / torch.sqrt(b.square().mean(1, keepdim=True) + EPS)
    n = wn * xo / torch.sqrt(xo.square().mean(1, keepdim=True) + EPS)
    out = {"x_out": xo.detach(), "n": n.detach()}
    if s["case"]["grad"]:
        d = torch.autograd.grad([xo, n], leaves, [s["dx_out"], s["dn"]])
        out.update(dx=d[0], db=d[1], dz=d[2], dw_post=d[3], dscale=d[4], dw_pre=d[5])
    return out


def _exact_orth(s):
    a, b, c = COEF
    m = None
    U = s.get("U")
    if U is None:
        m = s["momentum"] * BETA + s["grad"]
        U = m * BETA + s["grad"]
    X = U / torch.linalg.matrix_norm(U)[:, None, None]
    for _ in range(5):       # the polynomial X (a + b G + c G^2), by Horner, on the side with fewer products
        if X.shape[2] <= X.shape[1]:
            G = X.mT @ X
            Y = X @ G
            X = a * X + b * Y + c * (Y @ G)
        else:
            G = X @ X.mT
            Y = G @ X
            X = a * X + b * Y + c * (G @ Y)
    if m is None:
        return {"X": X}
    return {"W": s["W"] * (1 - LR * DECAY) - (LR * s["scale"]) * X, "momentum": m}
