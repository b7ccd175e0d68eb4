"""Performance cases of the expert layer that follows a router: the router's top-k choice is turned
into rows in expert order, every expert multiplies its rows, and the rows return to their tokens.

Kinds of case
  dispatch      ``Experts.sort`` and ``Experts.dispatch``: selections sorted by expert, tokens copied
                into expert order
  dispatch_bwd  ``Experts.dispatch_bwd``: the gradient of the tokens, the sum of their rows' gradients
                (plus the gradient that reached the tokens another way)
  combine       ``Experts.combine``: rows back to their tokens, weighted and summed, plus a residual
  combine_bwd   ``Experts.combine_bwd``: the gradients of the rows and of the weights
  linear        ``Experts.linear``: act(x W_e^T + b_e), gated or not, plus a residual
  act_bwd       ``Experts.act_bwd``: the gradients of the pre-activations and of the bias
  linear_bwd    ``Experts.linear_bwd``: the gradients of the rows and of the weights

A selection of -1 takes no part (a dropped or padding token); the rows that this leaves over at the
end of the expert order are zero. ``gated``: the pre-activations are two halves [g | u] of one row and
the output is act(g) * u.
"""
import math

import torch

DEV = "cuda"
own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
ACTS = {"none": 0, "silu": 1, "gelu": 2}


# ---------------------------------------------------------------------------------------- cases

def _tokens(kind, name, T, d, E, k, dtype="bf16", dropped=0.0, residual=False):
    c = dict(kind=kind, T=T, d=d, E=E, k=k, dtype=dtype, dropped=dropped, residual=residual)
    if name:
        c["name"] = name
    return c


def _product(kind, name, T, E, k, n_in, n_out, act="none", gated=False, bias=False, residual=False, pre=False,
             dtype="bf16", dropped=0.0):
    c = dict(kind=kind, T=T, E=E, k=k, n_in=n_in, n_out=n_out, act=act, gated=gated, bias=bias, residual=residual,
             pre=pre, dtype=dtype, dropped=dropped)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # serving: one decoding step of sixteen sequences through a dsmoe_vlm layer
        _tokens("dispatch", "decode_dispatch", 16, 2048, 64, 6),
        # the large_fine workload: 131072 tokens, eight of 128 experts each
        _tokens("dispatch", "large_dispatch", 131072, 2048, 128, 8),
        # fine-tuning on a small ragged batch with padding tokens: the router's own gradient of the
        # tokens joins that of the experts
        _tokens("dispatch_bwd", "ragged_dispatch_bwd", 6007, 1416, 48, 5, dropped=0.1, residual=True),
        # the dsmoe_vlm workload: the experts' rows back to the residual stream
        _tokens("combine", "dsmoe_combine", 16384, 2048, 64, 6, residual=True),
        # the small_hidden workload in training
        _tokens("combine_bwd", "small_hidden_combine_bwd", 32768, 1280, 64, 6),
        # the tiny_fp32 workload in training
        _tokens("combine_bwd", "tiny_fp32_combine_bwd", 4096, 512, 16, 2, dtype="fp32"),
        # serving: the decoding step's gated up-projection, bound by the weights it reads
        _product("linear", "decode_up", 16, 64, 6, 2048, 1024, act="silu", gated=True),
        # dsmoe_vlm in training: the gated up-projection, its pre-activations kept for the gradient
        _product("linear", "dsmoe_up", 16384, 64, 6, 2048, 1024, act="silu", gated=True, pre=True),
        # one shared expert of a small ragged batch: bias, activation and residual in one product
        _product("linear", "ragged_shared", 6007, 1, 1, 1416, 1416, act="gelu", bias=True, residual=True),
        # a ragged batch's up-projection with a bias: gradients of pre-activations and bias
        _product("act_bwd", "ragged_act_bwd", 6007, 48, 5, 1416, 704, act="silu", gated=True, bias=True, dropped=0.1),
        # dsmoe_vlm in training: the up-projection's gradients of rows and weights
        _product("linear_bwd", "dsmoe_up_bwd", 16384, 64, 6, 2048, 1024, gated=True),
        # tiny_fp32 in training
        _product("linear_bwd", "tiny_fp32_bwd", 4096, 16, 2, 512, 256, dtype="fp32"),
    ]


#: The largest listed cases: bytes of a data movement, flops of a product.
MOST_BYTES, MOST_FLOPS = 4.8e9, 1.6e12


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["dispatch", "dispatch_bwd", "combine", "combine_bwd", "linear", "linear", "linear", "act_bwd",
                       "linear_bwd", "linear_bwd"])
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    E, k = rng.choice([(8, 2), (16, 2), (32, 4), (48, 5), (64, 6), (64, 8), (72, 4), (128, 8), (128, 8)])
    dropped = rng.choice([0.0, 0.0, 0.1])
    width = lambda: rng.choice([1024, 1280, 2048, 8 * _log_int(rng, 16, 256), 8 * _log_int(rng, 16, 256)])  # noqa: E731
    if kind in ("dispatch", "dispatch_bwd", "combine", "combine_bwd"):
        d = width()
        T = _log_int(rng, 1, 131072 if dtype == "bf16" else 16384)
        c = _tokens(kind, None, T, d, E, k, dtype, dropped, kind in ("dispatch_bwd", "combine") and rng.random() < 0.6)
        while work(c)["bytes"] > MOST_BYTES:
            c["T"] //= 2
        return c
    if kind == "linear" and rng.random() < 0.25:        # a dense layer or a shared expert
        E, k, dropped = 1, 1, 0.0
    gated = rng.random() < 0.5
    act = rng.choice(["silu", "silu", "gelu"]) if gated or kind == "act_bwd" or rng.random() < 0.5 else "none"
    c = _product(kind, None, _log_int(rng, 1, 32768 if dtype == "bf16" else 4096), E, k, width(),
                 width() // (16 if gated else 8) * 8, act=act if kind != "linear_bwd" else "none", gated=gated,
                 bias=kind != "linear_bwd" and rng.random() < 0.5, residual=kind == "linear" and rng.random() < 0.4,
                 pre=kind == "linear" and act != "none" and rng.random() < 0.5, dtype=dtype, dropped=dropped)
    while work(c)["flops"] > (MOST_FLOPS if dtype == "bf16" else MOST_FLOPS / 16) or work(c)["bytes"] > MOST_BYTES:
        c["T"] //= 2
    return c


# --------------------------------------------------------------------------------------- inputs

def _n_z(c):
    return c["n_out"] * (2 if c["gated"] else 1)


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = TYPES[c["dtype"]]
    T, E, k = c["T"], c["E"], c["k"]
    R = T * k

    def normal(*shape, std=1.0, dtype=dt):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std).to(dtype)

    # a trained router's choice: some experts are liked better than others, some tokens are padding
    score = torch.randn((T, E), generator=g, device=DEV) + 0.5 * torch.randn(E, generator=g, device=DEV)
    top, idx = score.topk(k, dim=1)
    idx = idx.to(torch.int32)
    if c["dropped"]:
        idx[torch.rand(T, generator=g, device=DEV) < c["dropped"]] = -1
    s = dict(c=c, T=T, E=E, k=k, R=R, idx=idx.contiguous(), w=torch.softmax(top, 1))
    del score, top

    # the selections in expert order (stable: expert, then token, then slot): what the calls after
    # the sort have in hand
    flat = s["idx"].flatten()
    order = torch.sort(torch.where(flat < 0, E, flat), stable=True).indices.to(torch.int32)
    count = torch.bincount(flat[flat >= 0].long(), minlength=E)
    n = int(count.sum())
    s["offsets"] = torch.cat([count.new_zeros(1), count.cumsum(0)]).to(torch.int32)
    s["row_slot"] = torch.where(torch.arange(R, device=DEV) < n, order, -1)
    s["slot_row"] = torch.full((R,), -1, dtype=torch.int32, device=DEV)
    s["slot_row"][order[:n].long()] = torch.arange(n, dtype=torch.int32, device=DEV)
    s["slot_row"] = s["slot_row"].view(T, k)
    s["most"] = max(1, int(count.max()))                # rows of the largest expert, for the plain form's batches

    def rows(width, std=1.0):                           # rows in expert order; zero past the last selection
        x = normal(R, width, std=std)
        x[n:] = 0
        return x

    kind = c["kind"]
    if kind == "dispatch":
        s["X"] = normal(T, c["d"])
    elif kind == "dispatch_bwd":
        s["dXs"], s["residual"] = rows(c["d"]), normal(T, c["d"]) if c["residual"] else None
    elif kind == "combine":
        s["Ys"], s["residual"] = rows(c["d"]), normal(T, c["d"]) if c["residual"] else None
    elif kind == "combine_bwd":
        s["dY"], s["Ys"] = normal(T, c["d"]), rows(c["d"])
    elif kind == "linear":
        s["X"] = rows(c["n_in"])
        s["W"] = normal(E, _n_z(c), c["n_in"], std=c["n_in"] ** -0.5)
        s["bias"] = normal(E, _n_z(c), std=0.1, dtype=torch.float32) if c["bias"] else None
        s["residual"] = rows(c["n_out"]) if c["residual"] else None
    elif kind == "act_bwd":
        s["dOut"], s["pre"] = rows(c["n_out"]), rows(_n_z(c))
    else:
        s["dZ"], s["X"] = rows(_n_z(c)), rows(c["n_in"])
        s["W"] = normal(E, _n_z(c), c["n_in"], std=c["n_in"] ** -0.5)
    if own:                                             # the plan and workspace that a program keeps
        from paper_2604_23996_gb300 import binding as bd
        s["ex"] = bd.Experts(T, E, k, dtype=bd.SMOES_BF16 if dt is torch.bfloat16 else bd.SMOES_F32,
                             max_width=_n_z(c) if "n_out" in c else 0)
        if kind != "dispatch":
            s["ex"].sort(s["idx"])
    return s


# ------------------------------------------------------------------------------------------ run

def _run_own(s):
    c, ex = s["c"], s["ex"]
    kind = c["kind"]
    if kind == "dispatch":
        ex.sort(s["idx"])
        return {"offsets": ex.expert_offsets, "row_slot": ex.row_slot, "slot_row": ex.slot_row, "Xs": ex.dispatch(s["X"])}
    if kind == "dispatch_bwd":
        return {"dX": ex.dispatch_bwd(s["dXs"], residual=s["residual"])}
    if kind == "combine":
        return {"Y": ex.combine(s["Ys"], s["w"], residual=s["residual"])}
    if kind == "combine_bwd":
        dYs, dw = ex.combine_bwd(s["dY"], s["Ys"], s["w"])
        return {"dYs": dYs, "dw": dw}
    if kind == "linear":
        out, pre = ex.linear(s["X"], s["W"], bias=s["bias"], act=ACTS[c["act"]], gated=c["gated"],
                             residual=s["residual"], save_pre=c["pre"])
        return {"out": out, "pre": pre}
    if kind == "act_bwd":
        dZ, db = ex.act_bwd(s["dOut"], s["pre"], act=ACTS[c["act"]], gated=c["gated"], bias_grad=c["bias"])
        return {"dZ": dZ, "db": db}
    dX, dW = ex.linear_bwd(s["dZ"], s["X"], s["W"])
    return {"dX": dX, "dW": dW}


def _act(name, z):
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(name, z):
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5
    return torch.ones_like(z)


def _place(s):
    """Each row's expert and place among the expert's rows, and which rows there are."""
    r = torch.arange(s["R"], dtype=torch.int32, device=DEV)
    e = torch.searchsorted(s["offsets"], r, right=True) - 1
    there = e < s["E"]
    e = e.clamp(max=s["E"] - 1)
    return e, (r - s["offsets"][e]).clamp(max=s["most"] - 1).long(), there


def _batch(s, x, place):
    """Rows in expert order as one batch [E, most, width], zero where an expert has fewer."""
    e, i, there = place
    b = x.new_zeros((s["E"], s["most"], x.shape[1]), dtype=torch.float32)
    return b.index_put_((e[there], i[there]), x[there].float())


def _rows(s, b, place):
    e, i, there = place
    return b[e, i] * there[:, None]


def _taken(s, rows):
    """[T, k, width]: the row of each selection, zero for one that takes no part."""
    at = s["slot_row"].long()
    return rows.float()[at.clamp(min=0)] * (at >= 0)[..., None]


def _run_plain(s):
    c = s["c"]
    kind, dt = c["kind"], TYPES[c["dtype"]]
    if kind == "dispatch":
        flat = s["idx"].flatten()
        flat = torch.where(flat < 0, s["E"], flat)
        order = torch.sort(flat, stable=True).indices.to(torch.int32)
        r = torch.arange(s["R"], dtype=torch.int32, device=DEV)
        count = torch.zeros(s["E"] + 1, dtype=torch.int32, device=DEV).index_add_(0, flat, torch.ones_like(flat))
        offsets = torch.cat([count.new_zeros(1), count[:-1].cumsum(0, dtype=torch.int32)])
        there = r < offsets[-1]
        place = torch.empty_like(order).index_put_((order.long(),), r)
        Xs = s["X"].float()[order.long() // s["k"]] * there[:, None]
        return {"offsets": offsets, "row_slot": torch.where(there, order, -1),
                "slot_row": torch.where(place < offsets[-1], place, -1).view(s["T"], s["k"]), "Xs": Xs.to(dt)}
    if kind == "dispatch_bwd":
        dX = _taken(s, s["dXs"]).sum(1)
        return {"dX": (dX if s["residual"] is None else dX + s["residual"].float()).to(dt)}
    if kind == "combine":
        Y = (_taken(s, s["Ys"]) * s["w"][..., None]).sum(1)
        return {"Y": (Y if s["residual"] is None else Y + s["residual"].float()).to(dt)}
    if kind == "combine_bwd":
        dY = s["dY"].float()
        dw = (_taken(s, s["Ys"]) * dY[:, None, :]).sum(2)
        slot = s["row_slot"].long()
        w = torch.where(slot < 0, 0.0, s["w"].flatten()[slot.clamp(min=0)])
        return {"dYs": (dY[slot.clamp(min=0) // s["k"]] * w[:, None]).to(dt), "dw": dw}
    if kind == "act_bwd":
        z, d = s["pre"].float(), s["dOut"].float()
        if c["gated"]:
            a, u = z[:, :c["n_out"]], z[:, c["n_out"]:]
            dZ = torch.cat([d * u * _act_grad(c["act"], a), d * _act(c["act"], a)], 1)
        else:
            dZ = d * _act_grad(c["act"], z)
        return {"dZ": dZ.to(dt), "db": _batch(s, dZ, _place(s)).sum(1) if c["bias"] else None}
    place = _place(s)
    X, W = _batch(s, s["X"], place), s["W"].float()
    if kind == "linear":
        z = torch.bmm(X, W.transpose(1, 2))
        if s["bias"] is not None:
            z = z + s["bias"][:, None, :]
        z = _rows(s, z, place)
        y = _act(c["act"], z[:, :c["n_out"]])
        if c["gated"]:
            y = y * z[:, c["n_out"]:]
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"out": y.to(dt), "pre": z.to(dt) if c["pre"] else None}
    dZ = _batch(s, s["dZ"], place)
    return {"dX": _rows(s, torch.bmm(dZ, W), place).to(dt), "dW": torch.bmm(dZ.transpose(1, 2), X)}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ----------------------------------------------------------------------------------------- work

def work(c):
    b = 2 if c["dtype"] == "bf16" else 4
    T, E, k, kind = c["T"], c["E"], c["k"], c["kind"]
    R = T * k
    if "d" in c:
        d = c["d"]
        if kind == "dispatch":                          # selections, tokens; offsets, both maps, rows
            return {"bytes": 4 * R + b * T * d + 4 * (E + 1) + 8 * R + b * R * d, "flops": 0}
        if kind == "combine_bwd":                       # dY, rows, weights, maps; dYs, dw
            return {"bytes": b * T * d + b * R * d + 8 * R + b * R * d + 4 * R, "flops": 3 * R * d}
        return {"bytes": b * R * d + 4 * R * (2 if kind == "combine" else 1) + b * T * d * (2 if c["residual"] else 1),
                "flops": (2 if kind == "combine" else 1) * R * d}
    n_in, n_out, n_z = c["n_in"], c["n_out"], _n_z(c)
    # weights of the experts that have rows: with few tokens not all of them
    active = E * (1 - (1 - k / E) ** T) if E > 1 else 1
    if kind == "linear":
        return {"bytes": b * (R * n_in + active * n_z * n_in + R * n_out * (2 if c["residual"] else 1)
                              + (R * n_z if c["pre"] else 0)) + (4 * active * n_z if c["bias"] else 0),
                "flops": 2 * R * n_in * n_z}
    if kind == "act_bwd":
        return {"bytes": b * (R * n_out + 2 * R * n_z) + (4 * E * n_z if c["bias"] else 0), "flops": 8 * R * n_out}
    return {"bytes": b * (R * n_z + 2 * R * n_in + active * n_z * n_in) + 4 * E * n_z * n_in, "flops": 4 * R * n_in * n_z}


# ---------------------------------------------------------------------------------------- exact

def exact(c, seed):
    """The definitions token by token and expert by expert, in 64 bits."""
    s = prepare(c, seed)
    kind, E, k = c["kind"], c["E"], c["k"]
    if kind == "dispatch":                              # a copy: nothing is computed
        slot = s["row_slot"].long()
        Xs = s["X"].double().index_select(0, torch.div(slot.clamp(min=0), k, rounding_mode="floor"))
        Xs[slot < 0] = 0
        return {"offsets": None, "row_slot": None, "slot_row": None, "Xs": Xs}
    off = s["offsets"].tolist()
    if kind in ("dispatch_bwd", "combine", "combine_bwd"):
        rows = s["dXs" if kind == "dispatch_bwd" else "Ys"]
        T, d = s["T"], c["d"]
        if kind == "combine_bwd":
            dYs = torch.zeros(s["R"], d, dtype=torch.float64, device=DEV)
            dw = torch.zeros(T, k, dtype=torch.float64, device=DEV)
        else:
            out = s["residual"].double() if s.get("residual") is not None else torch.zeros(T, d, dtype=torch.float64, device=DEV)
        for j in range(k):
            at = s["slot_row"][:, j]
            t = torch.nonzero(at >= 0).flatten()
            at = at[t].long()
            if kind == "dispatch_bwd":
                out[t] += rows[at].double()
            elif kind == "combine":
                out[t] += s["w"][t, j].double().unsqueeze(1) * rows[at].double()
            else:
                g = s["dY"][t].double()
                dYs[at] = g * s["w"][t, j].double().unsqueeze(1)
                dw[t, j] = torch.einsum("td,td->t", g, rows[at].double())
        return {"dYs": dYs, "dw": dw} if kind == "combine_bwd" else {"Y" if kind == "combine" else "dX": out}
    n_out, n_z = c["n_out"], _n_z(c)

    def sigmoid(z):
        return torch.special.expit(z)

    def phi(z):                                         # the normal distribution's function
        return torch.special.ndtr(z)

    act = {"none": lambda z: z, "silu": lambda z: z * sigmoid(z), "gelu": lambda z: z * phi(z)}[c["act"]]
    slope = {"none": lambda z: torch.ones_like(z),
             "silu": lambda z: sigmoid(z) + z * sigmoid(z) * sigmoid(-z),
             "gelu": lambda z: phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[c["act"]]
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)  # noqa: E731
    if kind == "linear":
        out, pre = new(s["R"], n_out), new(s["R"], n_z) if c["pre"] else None
    elif kind == "act_bwd":
        dZ, db = new(s["R"], n_z), new(E, n_z) if c["bias"] else None
    else:
        dX, dW = new(s["R"], c["n_in"]), new(E, n_z, c["n_in"])
    for e in range(E):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        if kind == "linear":
            z = s["X"][a:b].double() @ s["W"][e].double().T
            if c["bias"]:
                z += s["bias"][e].double()
            out[a:b] = act(z[:, :n_out]) * (z[:, n_out:] if c["gated"] else 1.0)
            if c["residual"]:
                out[a:b] += s["residual"][a:b].double()
            if c["pre"]:
                pre[a:b] = z
        elif kind == "act_bwd":
            z, g = s["pre"][a:b].double(), s["dOut"][a:b].double()
            dZ[a:b, :n_out] = g * slope(z[:, :n_out]) * (z[:, n_out:] if c["gated"] else 1.0)
            if c["gated"]:
                dZ[a:b, n_out:] = g * act(z[:, :n_out])
            if c["bias"]:
                db[e] = dZ[a:b].sum(0)
        else:
            g = s["dZ"][a:b].double()
            dX[a:b] = g @ s["W"][e].double()
            dW[e] = g.T @ s["X"][a:b].double()
    if kind == "linear":
        return {"out": out, "pre": pre}
    if kind == "act_bwd":
        return {"dZ": dZ, "db": db}
    return {"dX": dX, "dW": dW}
