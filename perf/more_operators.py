"""Performance cases of what surrounds the router and the experts of one layer: the layer norm in front of them, the
expert-level balance loss of the router, and the experts' products of 4-bit microscaled values.

Kinds of case
  norm         ``LayerNorm.forward``: the residual stream's sum, its norm, the rows' statistics
  norm_bwd     ``LayerNorm.backward``: the gradients of the rows, of the weight and of the bias
  balance      ``Router.expert_balance``: the loss, the selections per expert, the gradient of the gate values (which is
               the same for all tokens of a sample, or of the batch)
  balance_bwd  the same, then ``Router.backward`` with it: the gradients of the logits, the gate weights and the tokens
  mx_values    ``mx_quantise`` and ``mx_dequantise``: values rounded to 4 bits in blocks of 32 with a common scale
  mx_linear    ``Experts.dispatch_mx`` (tokens quantised and copied into expert order) or ``mx_quantise`` (rows that are
               in expert order already), then ``Experts.linear_mx``: act(x W_e^T + b_e), gated or not, plus a residual

A selection of -1 takes no part. ``gated``: the pre-activations are two halves [g | u] of one row and the output is
act(g) * u. A block of 32 values has the scale 2^(floor(log2 of its largest) - 2); its values over the scale are rounded
to 0, 0.5, 1, 1.5, 2, 3, 4 or 6 with their sign, a tie to the even one of the eight, above 6 to 6.
"""
import math

import torch

DEV = "cuda"
own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
ACTS = {"none": 0, "silu": 1, "gelu": 2}
EPS = 1e-5


# ---------------------------------------------------------------------------------------- cases

def _case(kind, name, **values):
    c = dict(kind=kind, **values)
    if name:
        c["name"] = name
    return c


def _norm(kind, name, T, d, dtype="bf16", residual=False):
    return _case(kind, name, T=T, d=d, dtype=dtype, residual=residual)


def _balance(kind, name, T, d, E, k, samples, per_sample=True, dtype="bf16", dropped=0.0, gate="softmax"):
    return _case(kind, name, T=T, d=d, E=E, k=k, samples=samples, per_sample=per_sample, dtype=dtype, dropped=dropped,
                 gate=gate)


def _mx(name, T, E, k, n_in, n_out, dispatch, act="none", gated=False, bias=False, residual=False, dropped=0.0):
    return _case("mx_linear", name, T=T, E=E, k=k, n_in=n_in, n_out=n_out, dispatch=dispatch, act=act, gated=gated,
                 bias=bias, residual=residual, dropped=dropped, dtype="bf16")


def listed():
    return [
        # serving: one decoding step of sixteen sequences, the residual stream's sum and norm in one pass
        _norm("norm", "decode_norm", 16, 2048, residual=True),
        # the large_fine workload: 131072 tokens of the residual stream
        _norm("norm", "large_norm", 131072, 2048, residual=True),
        # dsmoe_vlm in training: the norm's gradients, the residual stream's own gradient added
        _norm("norm_bwd", "dsmoe_norm_bwd", 16384, 2048, residual=True),
        # a small ragged batch in fp32, at the width of the tiny_fp32 workload
        _norm("norm_bwd", "ragged_fp32_norm_bwd", 4091, 512, dtype="fp32"),
        # dsmoe_vlm in training: the loss of every sample
        _balance("balance", "dsmoe_balance", 16384, 2048, 64, 6, 8),
        # large_fine in training: the loss of the whole batch, some tokens are padding
        _balance("balance", "large_balance", 131072, 2048, 128, 8, 32, per_sample=False, dropped=0.1),
        # small_hidden in training: the loss and its way back to gate weights and tokens
        _balance("balance_bwd", "small_hidden_balance_bwd", 32768, 1280, 64, 6, 16),
        # the down-projections of the dsmoe_vlm layer, quantised for serving and read back
        _case("mx_values", "dsmoe_weight_values", rows=64 * 2048, n=1024, dtype="bf16"),
        # serving: the decoding step's gated up-projection, bound by the weights it reads
        _mx("decode_mx_up", 16, 64, 6, 2048, 1024, True, act="silu", gated=True),
        # serving: prompts of 16384 tokens through dsmoe_vlm's gated up-projection
        _mx("dsmoe_mx_up", 16384, 64, 6, 2048, 1024, True, act="silu", gated=True),
        # and back: its down-projection of rows that are in expert order already
        _mx("dsmoe_mx_down", 16384, 64, 6, 1024, 2048, False),
        # a shared expert on a small ragged batch: bias, activation and residual in one product
        _mx("ragged_mx_shared", 6007, 1, 1, 1440, 1416, True, act="gelu", bias=True, residual=True),
    ]


#: The largest listed cases: bytes of what moves data, flops and weights of a product.
MOST_BYTES, MOST_FLOPS, MOST_WEIGHTS = 2.1e9, 8.2e11, 64 * 2048 * 2048


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "balance", "balance_bwd", "mx_values", "mx_linear", "mx_linear", "mx_linear"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if kind in ("norm", "norm_bwd"):
        c = _norm(kind, None, _log_int(rng, 1, 131072), 8 * _log_int(rng, 4, 1024), dtype, rng.random() < 0.5)
        while work(c)["bytes"] > MOST_BYTES:
            c["T"] //= 2
        return c
    if kind in ("balance", "balance_bwd"):
        E, k = rng.choice([(8, 2), (16, 2), (32, 4), (48, 5), (64, 6), (64, 8)] + [(72, 4), (128, 8)] * (dtype == "bf16"))
        T = _log_int(rng, 16, 131072 if kind == "balance" else 32768)
        return _balance(kind, None, T, rng.choice([512, 1280, 2048, 8 * _log_int(rng, 16, 256)]) if kind == "balance_bwd" else 256,
                        E, k, min(T, _log_int(rng, 1, 64)), rng.random() < 0.6, dtype, rng.choice([0.0, 0.0, 0.1]),
                        rng.choice(["softmax", "softmax", "sigmoid"]))
    if kind == "mx_values":
        n = 32 * _log_int(rng, 1, 128)
        return _case(kind, None, rows=_log_int(rng, 1, 134217728 // n), n=n, dtype=dtype)
    E, k, dropped = rng.choice([(8, 2, 0.0), (16, 2, 0.1), (32, 4, 0.0), (48, 5, 0.1), (64, 6, 0.0), (128, 8, 0.0), (1, 1, 0.0)])
    gated = rng.random() < 0.5
    c = _mx(None, _log_int(rng, 1, 16384), E, k, rng.choice([1024, 2048, 32 * _log_int(rng, 2, 128)]),
            rng.choice([1024, 1280, 8 * _log_int(rng, 16, 256)]), rng.random() < 0.5,
            act=rng.choice(["silu", "gelu"]) if gated else rng.choice(["none", "none", "silu", "gelu"]), gated=gated,
            bias=rng.random() < 0.3, residual=rng.random() < 0.3, dropped=dropped)
    while E * _n_z(c) * c["n_in"] > MOST_WEIGHTS:
        c["n_in"] = max(32, c["n_in"] // 64 * 32)
    while work(c)["flops"] > MOST_FLOPS or work(c)["bytes"] > MOST_BYTES:
        c["T"] //= 2
    return c


# --------------------------------------------------------------------------------------- inputs

def _n_z(c):
    return c["n_out"] * (2 if c["gated"] else 1)


def _quantised(x):
    """fp32 values [..., n] as pairs of 4-bit codes [..., n / 2] (the even one in the low half) and scale bytes [..., n / 32]."""
    b = x.reshape(-1, 32)
    exponent = (torch.frexp(b.abs().amax(1))[1] - 3).clamp(min=-127)          # frexp: 0.5 <= mantissa < 1
    a = torch.ldexp(b.abs(), -exponent[:, None])
    code = torch.zeros(b.shape, dtype=torch.int32, device=x.device)
    # half way between neighbours; a tie goes up where the upper one's code is even
    for i, edge in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += a >= edge if i % 2 else a > edge
    code += 8 * torch.signbit(b)
    pairs = code.view(-1, 16, 2)
    return ((pairs[..., 0] + 16 * pairs[..., 1]).to(torch.uint8).view(*x.shape[:-1], -1),
            (exponent + 127).to(torch.uint8).view(*x.shape[:-1], -1))


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = TYPES[c["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std).to(dtype)

    s = dict(c=c)
    kind = c["kind"]
    if own:
        from paper_2604_23996_gb300 import binding as bd
        code = bd.SMOES_BF16 if dt is torch.bfloat16 else bd.SMOES_F32
        s["bd"] = bd
    if kind in ("norm", "norm_bwd"):
        T, d = c["T"], c["d"]
        # a residual stream: tokens of different lengths, features of different means
        s["X"] = (normal(T, d, dtype=torch.float32) * (0.5 + torch.rand(T, 1, generator=g, device=DEV))
                  + 0.3 * normal(d, dtype=torch.float32)).to(dt)
        s["residual"] = normal(T, d) if c["residual"] else None
        s["w"] = 1 + 0.1 * normal(d, dtype=torch.float32)
        s["b"] = 0.1 * normal(d, dtype=torch.float32)
        if kind == "norm_bwd":                          # the forward's sum is X; the stream's gradient joins dX
            s["dY"] = normal(T, d)
            x = s["X"].double()
            mean = x.mean(1)
            s["mean"] = mean.float()
            s["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt().float()
        if own:
            s["norm"] = bd.LayerNorm(T, d, code, eps=EPS)
        return s
    if kind in ("balance", "balance_bwd"):
        T, d, E, k, B = c["T"], c["d"], c["E"], c["k"], c["samples"]
        cut = torch.linspace(0, T, B + 1, dtype=torch.float64).round().long()
        if B > 1:                                       # ragged samples, none of them empty
            shift = (torch.rand(B - 1, generator=g, device=DEV).cpu() - 0.5) * 0.8 * (T / B)
            cut[1:-1] = torch.maximum(torch.minimum(cut[1:-1] + shift.long(), T - torch.arange(B - 1, 0, -1)), torch.arange(1, B))
            cut = torch.cummax(cut, 0).values
            for i in range(1, B):
                cut[i] = max(int(cut[i]), int(cut[i - 1]) + 1)
        s["offsets"] = cut.to(DEV)
        s["sample"] = torch.repeat_interleave(torch.arange(B, device=DEV), s["offsets"].diff())
        # a router that likes some experts better than others
        s["X"] = normal(T, d)
        s["W"] = normal(E, d, std=d ** -0.5)
        s["score_bias"] = normal(E, std=0.1, dtype=torch.float32) if c["gate"] == "sigmoid" else None
        z = s["X"].float() @ s["W"].float().T
        s["raw"] = torch.sigmoid(z) if c["gate"] == "sigmoid" else torch.softmax(z, 1)
        s["gate"] = s["raw"] / s["raw"].sum(1, keepdim=True)
        pick = s["raw"] if s["score_bias"] is None else s["raw"] + s["score_bias"]
        s["idx"] = pick.topk(k, dim=1).indices.to(torch.int32)
        if c["dropped"]:
            s["idx"][torch.rand(T, generator=g, device=DEV) < c["dropped"]] = -1
        s["M"] = torch.full((T, 2), 0.5, device=DEV)
        if own:
            s["router"] = bd.Router(T, d, E, k, 1 if E <= 32 else E // 8, cut.tolist(),
                                    [0] * E if E <= 32 else [e // 8 for e in range(E)], code,
                                    gate=bd.SMOES_GATE_SIGMOID if c["gate"] == "sigmoid" else bd.SMOES_GATE_SOFTMAX,
                                    score_bias=s["score_bias"])
            s["router"].forward(s["X"], s["W"], M_in=s["M"])
            if kind == "balance_bwd":
                s["dW"] = torch.empty((E, d), dtype=torch.float32, device=DEV)
                s["dX"] = torch.empty((T, d), dtype=dt, device=DEV)
                s["dlogits"] = torch.empty((T, E), dtype=torch.float32, device=DEV)
        return s
    if kind == "mx_values":
        s["X"] = normal(c["rows"], c["n"], std=c["n"] ** -0.5)
        return s
    T, E, k = c["T"], c["E"], c["k"]
    R = T * k
    score = torch.randn((T, E), generator=g, device=DEV) + 0.5 * torch.randn(E, generator=g, device=DEV)
    idx = score.topk(k, dim=1).indices.to(torch.int32)
    if c["dropped"]:
        idx[torch.rand(T, generator=g, device=DEV) < c["dropped"]] = -1
    # the selections in expert order, as the sort leaves them
    flat = idx.flatten().long()
    order = torch.sort(torch.where(flat < 0, E, flat), stable=True).indices
    count = torch.bincount(flat[flat >= 0], minlength=E)
    n = int(count.sum())
    s["offsets"] = torch.cat([count.new_zeros(1), count.cumsum(0)])
    s["token"] = torch.where(torch.arange(R, device=DEV) < n, torch.div(order, k, rounding_mode="floor"), -1)
    s["most"] = max(1, int(count.max()))                # rows of the largest expert, for the plain form's batches
    s["X"] = normal(T if c["dispatch"] else R, c["n_in"])
    if not c["dispatch"]:
        s["X"][n:] = 0
    s["W"], s["W_scale"] = _quantised(normal(E, _n_z(c), c["n_in"], std=c["n_in"] ** -0.5, dtype=torch.float32))
    s["bias"] = normal(E, _n_z(c), std=0.1, dtype=torch.float32) if c["bias"] else None
    s["residual"] = normal(R, c["n_out"]) if c["residual"] else None
    if c["residual"]:
        s["residual"][n:] = 0
    if own:
        s["ex"] = bd.Experts(T, E, k, code)
        s["ex"].sort(idx.contiguous())
    return s


# ------------------------------------------------------------------------------------------ run

def _run_own(s):
    c, bd = s["c"], s["bd"]
    kind = c["kind"]
    if kind == "norm":
        Y, S, mean, rstd = s["norm"].forward(s["X"], s["w"], s["b"], residual=s["residual"])
        return {"Y": Y, "S": S if c["residual"] else None, "mean": mean, "rstd": rstd}
    if kind == "norm_bwd":
        dX, dw, db = s["norm"].backward(s["dY"], s["X"], s["mean"], s["rstd"], s["w"], residual=s["residual"])
        return {"dX": dX, "dw": dw, "db": db}
    if kind in ("balance", "balance_bwd"):
        r = s["router"]
        loss, counts, d_gate = r.expert_balance(topk_idx=s["idx"], per_sample=c["per_sample"], loss_scale=0.5)
        out = {"loss": loss, "counts": counts, "d_gate": d_gate}
        if kind == "balance_bwd":
            r.backward(s["X"], s["W"], s["M"], s["dW"], dX=s["dX"], dlogits=s["dlogits"], loss_scale=0.0, d_gate=d_gate,
                       topk_idx=s["idx"])
            out |= {"dW": s["dW"], "dX": s["dX"], "dlogits": s["dlogits"]}
        return out
    if kind == "mx_values":
        return {"values": bd.mx_dequantise(bd.mx_quantise(s["X"]))}
    ex = s["ex"]
    X = ex.dispatch_mx(s["X"]) if c["dispatch"] else bd.mx_quantise(s["X"])
    return {"out": ex.linear_mx(X, bd.Mx(s["W"], s["W_scale"]), bias=s["bias"], act=ACTS[c["act"]], gated=c["gated"],
                                residual=s["residual"])}


def _values(codes, scale):
    """fp32 values of pairs of 4-bit codes and their scale bytes."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    size = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)[(code & 7).long()]
    size = torch.where(code >= 8, -size, size)
    return (size.unflatten(-1, (-1, 32)) * torch.exp2(scale.float() - 127)[..., None]).flatten(-2)


def _rounded(x):
    """Values rounded to 4 bits with a scale for every 32 of them."""
    b = x.float().unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    exponent = torch.frexp(most)[1] - 3
    scale = torch.exp2(exponent.clamp(min=-127).float())
    a = b.abs() / scale
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.copysign((torch.round(a / step) * step).clamp(max=6.0), b) * scale).flatten(-2)


def _act(name, z):
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _run_plain(s):
    c = s["c"]
    kind, dt = c["kind"], TYPES[c["dtype"]]
    if kind == "norm":
        x = s["X"].float()
        S = None
        if s["residual"] is not None:
            S = (x + s["residual"].float()).to(dt)
            x = S.float()
        mean = x.sum(1) / c["d"]
        xc = x - mean[:, None]
        rstd = 1 / torch.sqrt((xc * xc).sum(1) / c["d"] + EPS)
        return {"Y": (xc * rstd[:, None] * s["w"] + s["b"]).to(dt), "S": S, "mean": mean, "rstd": rstd}
    if kind == "norm_bwd":
        dy = s["dY"].float()
        xh = (s["X"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        dxh = dy * s["w"]
        dx = s["rstd"][:, None] * (dxh - dxh.sum(1, keepdim=True) / c["d"] - xh * ((dxh * xh).sum(1, keepdim=True) / c["d"]))
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        return {"dX": dx.to(dt), "dw": (dy * xh).sum(0), "db": dy.sum(0)}
    if kind in ("balance", "balance_bwd"):
        E, B = c["E"], c["samples"] if c["per_sample"] else 1
        smp = s["sample"] if c["per_sample"] else torch.zeros_like(s["sample"])
        idx = s["idx"]
        taken = idx >= 0
        at = (smp[:, None] * E + idx)[taken]
        counts = torch.zeros(B * E, dtype=torch.int32, device=DEV).index_add_(0, at, torch.ones_like(at, dtype=torch.int32)).view(B, E)
        there = taken.any(1)
        n = torch.zeros(B, device=DEV).index_add_(0, smp, there.float())[:, None]
        f = E * counts / counts.sum(1, keepdim=True).clamp(min=1)
        P = torch.zeros(B, E, device=DEV).index_add_(0, smp, s["gate"] * there[:, None]) / n.clamp(min=1)
        d_gate = torch.where(n > 0, 0.5 * f / (B * n.clamp(min=1)), 0.0)
        out = {"loss": (f * P).sum().view(1) / B, "counts": counts, "d_gate": d_gate}
        if kind == "balance_bwd":
            t, g = d_gate[smp], s["gate"]
            dz = g * (t - (g * t).sum(1, keepdim=True)) * there[:, None]
            if c["gate"] == "sigmoid":
                dz = dz * (1 - s["raw"])
            out |= {"dW": dz.T @ s["X"].float(), "dX": (dz @ s["W"].float()).to(dt), "dlogits": dz}
        return out
    if kind == "mx_values":
        return {"values": _rounded(s["X"]).to(torch.bfloat16)}
    rows = _rounded(s["X"])
    token, E, off = s["token"], c["E"], s["offsets"]
    there = token >= 0
    if c["dispatch"]:
        rows = rows[token.clamp(min=0)]
    r = torch.arange(token.numel(), device=DEV)
    e = (torch.searchsorted(off, r, right=True) - 1).clamp(max=E - 1)
    i = (r - off[e]).clamp(max=s["most"] - 1)
    X = torch.zeros(E, s["most"], c["n_in"], device=DEV).index_put_((e[there], i[there]), rows[there])
    z = torch.bmm(X, _values(s["W"], s["W_scale"]).transpose(1, 2))
    if s["bias"] is not None:
        z = z + s["bias"][:, None, :]
    z = z[e, i] * there[:, None]
    y = _act(c["act"], z[:, :c["n_out"]])
    if c["gated"]:
        y = y * z[:, c["n_out"]:]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"out": y.to(dt)}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ----------------------------------------------------------------------------------------- work

def work(c):
    b = 2 if c["dtype"] == "bf16" else 4
    kind = c["kind"]
    if kind == "norm":                                  # X (and the residual), w, b; Y (and the sum), two statistics a row
        return {"bytes": b * c["T"] * c["d"] * (4 if c["residual"] else 2) + 8 * c["d"] + 8 * c["T"], "flops": 8 * c["T"] * c["d"]}
    if kind == "norm_bwd":                              # dY, X (and the residual's), statistics, w; dX, dw, db
        return {"bytes": b * c["T"] * c["d"] * (4 if c["residual"] else 3) + 8 * c["T"] + 12 * c["d"], "flops": 14 * c["T"] * c["d"]}
    if kind in ("balance", "balance_bwd"):              # gate values, selections; counts, gradient
        T, E, d = c["T"], c["E"], c["d"]
        table = (c["samples"] if c["per_sample"] else 1) * E
        w = {"bytes": 4 * T * E + 4 * T * c["k"] + 8 * table + 4, "flops": 2 * T * E}
        if kind == "balance_bwd":                       # and tokens, weights; dX, dW, dlogits
            w["bytes"] += 2 * b * (T * d) + b * E * d + 4 * E * d + 4 * T * E
            w["flops"] += 4 * T * E * d + 5 * T * E
        return w
    if kind == "mx_values":
        return {"bytes": c["rows"] * c["n"] * (b + 2), "flops": 4 * c["rows"] * c["n"]}
    T, E, k, n_in, n_out, n_z = c["T"], c["E"], c["k"], c["n_in"], c["n_out"], _n_z(c)
    R = T * k
    # weights of the experts that have rows: with few tokens not all of them
    active = E * (1 - (1 - k / E) ** T) if E > 1 else 1
    return {"bytes": 2 * (T if c["dispatch"] else R) * n_in + 17 / 32 * active * n_z * n_in
                     + 2 * R * n_out * (2 if c["residual"] else 1) + (4 * active * n_z if c["bias"] else 0),
            "flops": 2 * R * n_in * n_z}


# ---------------------------------------------------------------------------------------- exact

def _nearest(x):
    """Blocks of 32 rounded to the nearest of the values a block can hold, by looking at all of them, in 64 bits."""
    sizes = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    for a in range(0, x.shape[0], 65536):
        b = x[a:a + 65536].double().unflatten(-1, (-1, 32))
        top = b.abs().amax(-1, keepdim=True)
        scale = 2.0 ** (torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 2).clamp(min=-127)
        v = b.abs() / scale
        best, held = torch.full_like(v, math.inf), torch.zeros_like(v)
        for i in (0, 2, 4, 6, 1, 3, 5, 7):              # even ones first: they keep a tie
            off = (v - sizes[i]).abs()
            held = torch.where(off < best, sizes[i], held)
            best = torch.minimum(best, off)
        out[a:a + 65536] = (torch.sign(b) * held * scale).flatten(-2)
    return out


def exact(c, seed):
    """The definitions sample by sample and expert by expert, in 64 bits."""
    s = prepare(c, seed)
    kind = c["kind"]
    if kind in ("norm", "norm_bwd"):
        x, w = s["X"].double(), s["w"].double()
        if kind == "norm":
            S = None
            if c["residual"]:
                S = x + s["residual"].double()
                x = S.to(TYPES[c["dtype"]]).double()    # the norm is of the stream as it is kept
            mean, var = x.mean(1, keepdim=True), x.var(1, unbiased=False, keepdim=True)
            xh = (x - mean) / (var + EPS).sqrt()
            return {"Y": xh * w + s["b"].double(), "S": S, "mean": mean.flatten(), "rstd": 1 / (var + EPS).sqrt().flatten()}
        dy, rstd = s["dY"].double(), s["rstd"].double()[:, None]
        xh = (x - s["mean"].double()[:, None]) * rstd
        a = dy * w
        dx = a.sub(a.mean(1, keepdim=True)).sub(xh * torch.einsum("td,td->t", a, xh)[:, None] / c["d"]) * rstd
        if c["residual"]:
            dx += s["residual"].double()
        return {"dX": dx, "dw": torch.einsum("td,td->d", dy, xh), "db": dy.sum(0)}
    if kind in ("balance", "balance_bwd"):
        E, T = c["E"], c["T"]
        z = s["X"].double() @ s["W"].double().T
        raw = torch.special.expit(z) if c["gate"] == "sigmoid" else torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
        g = raw / raw.sum(1, keepdim=True)
        cut = s["offsets"].tolist() if c["per_sample"] else [0, T]
        B = len(cut) - 1
        loss = torch.zeros(1, dtype=torch.float64, device=DEV)
        d_gate = torch.zeros(B, E, dtype=torch.float64, device=DEV)
        dz = torch.zeros(T, E, dtype=torch.float64, device=DEV)
        for i in range(B):
            idx = s["idx"][cut[i]:cut[i + 1]].long()
            on = (idx >= 0).any(1)
            n = int(on.sum())
            if n == 0:
                continue
            share = torch.bincount(idx[idx >= 0], minlength=E).double()
            share *= E / share.sum()
            gi = g[cut[i]:cut[i + 1]] * on[:, None]
            loss += share @ gi.sum(0) / n / B
            d_gate[i] = 0.5 * share / (B * n)
            dz[cut[i]:cut[i + 1]] = gi * (d_gate[i] - (gi @ d_gate[i])[:, None])
        out = {"loss": loss, "counts": None, "d_gate": d_gate}
        if kind == "balance_bwd":
            if c["gate"] == "sigmoid":
                dz *= torch.special.expit(-z)
            out |= {"dW": dz.T @ s["X"].double(), "dX": dz @ s["W"].double(), "dlogits": dz}
        return out
    if kind == "mx_values":
        return {"values": _nearest(s["X"])}
    E, n_out = c["E"], c["n_out"]
    X = _nearest(s["X"])
    sizes = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    sizes = torch.tensor(sizes + [-v for v in sizes], dtype=torch.float64, device=DEV)
    act = {"none": lambda z: z, "silu": lambda z: z * torch.special.expit(z), "gelu": lambda z: z * torch.special.ndtr(z)}[c["act"]]
    out = torch.zeros(s["token"].numel(), n_out, dtype=torch.float64, device=DEV)
    off = s["offsets"].tolist()
    for e in range(E):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        W = torch.empty(_n_z(c), c["n_in"], dtype=torch.float64, device=DEV)
        W[:, 0::2] = sizes[(s["W"][e] % 16).long()]
        W[:, 1::2] = sizes[torch.div(s["W"][e], 16, rounding_mode="floor").long()]
        W *= (2.0 ** (s["W_scale"][e].double() - 127)).repeat_interleave(32, 1)
        z = (X[s["token"][a:b]] if c["dispatch"] else X[a:b]) @ W.T
        if c["bias"]:
            z += s["bias"][e].double()
        out[a:b] = act(z[:, :n_out]) * (z[:, n_out:] if c["gated"] else 1.0)
        if c["residual"]:
            out[a:b] += s["residual"][a:b].double()
    return {"out": out}
