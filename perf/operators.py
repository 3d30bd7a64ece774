"""Performance cases of the 8-bit integer feed-forward path: the root-mean-square norm that ends in codes, the gated
activation that ends in codes, the product of codes with scales for each token and channel, the mixture-of-experts layer
for a few tokens, and the gradients of the first two.

`own` False: every operator in its plain form, elementary torch operations in fp32; True: the package's entry points.

Codes are int8 with one fp32 scale a row.  Outputs that are held as codes are returned as the values they stand for,
code * scale in bfloat16 (an 8-bit code has no more digits than that), with the scales beside them.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_EPS = 1e-5


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # One token of a serving step: residual addition, norm and quantization in front of a product of width 4096.
        dict(name="norm_token", kind="norm", rows=1, width=4096, type="bf16", residual=True),
        # The same in front of a prefill of 10 000 tokens.
        dict(name="norm_10000", kind="norm", rows=10000, width=4096, type="bf16", residual=True),
        # Gradient of that norm in a training step, with the gradient of the residual path joined in.
        dict(name="norm_grad_10000", kind="norm_grad", rows=10000, width=4096, type="bf16", residual=True),
        # The same in full precision, ragged batch and a width that is no multiple of anything large; no residual path.
        dict(name="norm_grad_odd", kind="norm_grad", rows=1999, width=2500, type="f32", residual=False),
        # Gated activation between the two products of a block, prefill of 10 000 tokens.
        dict(name="gate_10000", kind="gate", rows=10000, width=4096, type="bf16"),
        # Its gradient, over a training window of 2240 tokens, odd width.
        dict(name="gate_grad_odd", kind="gate_grad", rows=2240, width=2501, type="f16"),
        # One token through a layer of 4096 x 4096 8-bit weights.
        dict(name="product_token", kind="product", m=1, n=4096, k=4096, type="bf16", bias=False),
        # A product of no convenient size, with a bias.
        dict(name="product_odd", kind="product", m=1999, n=3001, k=2500, type="f32", bias=True),
        # The large product: a prefill of 8192 tokens through a square layer.
        dict(name="product_8192", kind="product", m=8192, n=8192, k=8192, type="bf16", bias=False),
        # One token through a layer of 8 experts, two chosen.
        dict(name="moe_token", kind="moe", tokens=1, experts=8, top=2, hidden=4096, inner=2048, type="bf16"),
        # A serving batch of 20 tokens through the same layer.
        dict(name="moe_batch", kind="moe", tokens=20, experts=8, top=2, hidden=4096, inner=2048, type="bf16"),
        # A few tokens, odd widths, an odd number of experts.
        dict(name="moe_odd", kind="moe", tokens=7, experts=5, top=3, hidden=1000, inner=700, type="f32"),
    ]


def _log_int(rng, lo, hi):
    v = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return v + (v == 3072)  # (no configuration here has that size)


def _width(rng, lo, hi):
    """A width: a multiple of 64 half of the time, any number otherwise."""
    v = _log_int(rng, lo, hi)
    even = max(lo, v // 64 * 64)
    return even if rng.random() < 0.5 and even != 3072 else v


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "gate", "gate_grad", "product", "product", "product", "moe", "moe"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("norm", "norm_grad"):
        return dict(kind=kind, rows=_log_int(rng, 1, 10000), width=_width(rng, 64, 4096), type=t, residual=rng.random() < 0.7)
    if kind in ("gate", "gate_grad"):
        return dict(kind=kind, rows=_log_int(rng, 1, 10000), width=_width(rng, 64, 4096), type=t)
    if kind == "product":
        return dict(kind=kind, m=_log_int(rng, 1, 8192), n=_width(rng, 64, 8192), k=_width(rng, 64, 8192), type=t,
                    bias=rng.random() < 0.3)
    experts = rng.randint(2, 16)
    return dict(kind=kind, tokens=_log_int(rng, 1, 32), experts=experts, top=rng.randint(1, min(4, experts)),
                hidden=_width(rng, 256, 4096), inner=_width(rng, 128, 1024), type=t)


# ------------------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _uniform(g, lo, hi, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32) * (hi - lo) + lo


def _codes(g, *shape):
    """Codes of normally distributed values whose largest is four deviations."""
    return _normal(g, *shape).mul_(32).round_().clamp_(-127, 127).to(torch.int8)


def _inputs(case, seed):
    """Inputs of a case, on the GPU, from the seed alone."""
    g, kind, t = _gen(seed), case["kind"], _TYPES[case["type"]]
    if kind in ("norm", "norm_grad"):
        rows, k = case["rows"], case["width"]
        channel = torch.exp(_normal(g, k) * 0.5)  # channels of a residual stream differ in size
        d = dict(x=(_normal(g, rows, k) * channel).to(t), gamma=(1 + 0.1 * _normal(g, k)).to(t))
        if kind == "norm_grad":
            d["grad"] = (_normal(g, rows, k) * 0.1).to(t)
        if case["residual"]:
            d["residual"] = (_normal(g, rows, k) * (0.1 if kind == "norm_grad" else 2)).to(t)
        return d
    if kind in ("gate", "gate_grad"):
        rows, f = case["rows"], case["width"]
        d = dict(u=_normal(g, rows, 2 * f).mul_(1.5).to(t))  # as a product leaves it: gate and up side by side
        if kind == "gate_grad":
            d["grad"] = (_normal(g, rows, f) * 0.1).to(t)
        return d
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        d = dict(a=_codes(g, m, k), sa=_uniform(g, 0.01, 0.04, m), w=_codes(g, n, k), sw=_uniform(g, 0.0005, 0.001, n))
        if case["bias"]:
            d["bias"] = _normal(g, n) * 0.1
        return d
    tk, e, h, f = case["tokens"], case["experts"], case["hidden"], case["inner"]
    return dict(x=_codes(g, tk, h), sx=_uniform(g, 0.01, 0.04, tk), logits=_normal(g, tk, e),
                w1=_codes(g, e, 2 * f, h), s1=_uniform(g, 0.0005, 0.001, e, 2 * f),
                w2=_codes(g, e, h, f), s2=_uniform(g, 0.0005, 0.001, e, h))


def prepare(case, seed):
    """Inputs, weights, and the outputs and workspaces that a program keeps between calls."""
    d, kind, t = _inputs(case, seed), case["kind"], _TYPES[case["type"]]
    new = lambda *shape, dtype=t: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    st = dict(case=case, **d)
    if kind in ("norm", "gate"):
        rows, k = case["rows"], case["width"]
        st.update(codes=new(rows, k, dtype=torch.int8), scale=new(rows, dtype=torch.float32), values=new(rows, k, dtype=torch.bfloat16))
        if kind == "norm" and case["residual"]:
            st["total"] = new(rows, k)
    elif kind == "norm_grad":
        # (partial sums of the weight's gradient: a few hundred rows)
        st.update(out=new(case["rows"], case["width"]), gw=new(case["width"], dtype=torch.float32),
                  ws=new(1 << 23, dtype=torch.uint8))
    elif kind == "gate_grad":
        st["out"] = new(case["rows"], 2 * case["width"])
    elif kind == "product":
        st["out"] = new(case["m"], case["n"])
    else:
        # (activations between the two products in fp32, and their maxima)
        st.update(out=new(case["tokens"], case["hidden"]),
                  ws=new(case["tokens"] * case["top"] * (8 * case["inner"] + 4096) + 65536, dtype=torch.uint8))
    return st


# ------------------------------------------------------------------------------------------------------- plain forms
def _quantize(y):
    """(codes as fp32, scales) of every row."""
    scale = y.abs().amax(dim=-1, keepdim=True) / 127
    return torch.where(scale > 0, torch.round(y / scale), 0.0), scale


def _values(y):
    codes, scale = _quantize(y)
    return (codes * scale).to(torch.bfloat16), scale[:, 0]


def _silu(x):
    return x / (1 + torch.exp(-x))


def _norm(s):
    t, h = s["x"].dtype, s["x"].float()
    if s["case"]["residual"]:
        h = h + s["residual"].float()
    r = torch.rsqrt((h * h).mean(dim=-1, keepdim=True) + _EPS)
    values, scale = _values(h * r * s["gamma"].float())
    return [values, scale] + ([h.to(t)] if s["case"]["residual"] else [])


def _norm_grad(s):
    t, h, g, w = s["x"].dtype, s["x"].float(), s["grad"].float(), s["gamma"].float()
    r = torch.rsqrt((h * h).mean(dim=-1, keepdim=True) + _EPS)
    wg = g * w
    gh = r * (wg - h * (r * r) * (wg * h).mean(dim=-1, keepdim=True))
    if s["case"]["residual"]:
        gh = gh + s["residual"].float()
    return [gh.to(t), (g * h * r).sum(dim=0)]


def _gate(s):
    f = s["case"]["width"]
    u = s["u"].float()
    return list(_values(_silu(u[:, :f]) * u[:, f:]))


def _gate_grad(s):
    f = s["case"]["width"]
    u, g = s["u"].float(), s["grad"].float()
    gate, up = u[:, :f], u[:, f:]
    p = 1 / (1 + torch.exp(-gate))
    return torch.cat([g * up * p * (1 + gate * (1 - p)), g * gate * p], dim=1).to(s["u"].dtype)


def _product(s):
    y = (s["a"].float() @ s["w"].float().t()) * s["sa"][:, None] * s["sw"]
    if s["case"]["bias"]:
        y = y + s["bias"]
    return y.to(s["out"].dtype)


def _moe(s):
    c = s["case"]
    tk, k, f = c["tokens"], c["top"], c["inner"]
    order = torch.sort(s["logits"], dim=-1, descending=True, stable=True)
    ids, p = order.indices[:, :k], torch.exp(order.values[:, :k] - order.values[:, :1])
    p = p / p.sum(dim=-1, keepdim=True)
    x = s["x"].float() * s["sx"][:, None]
    if tk * k <= c["experts"]:  # the chosen experts' weights, by token and choice
        w1, w2, s1, s2 = s["w1"][ids].float(), s["w2"][ids].float(), s["s1"][ids], s["s2"][ids]
        u = (w1 @ x[:, None, :, None])[..., 0] * s1
        a, sa = _quantize(_silu(u[..., :f]) * u[..., f:])
        v = (w2 @ (a * sa)[..., None])[..., 0] * s2
        return (v * p[..., None]).sum(dim=1).to(s["out"].dtype)
    # every expert for every token, weighted with zero where it is not chosen
    u = torch.matmul(x, s["w1"].float().transpose(1, 2)) * s["s1"][:, None]
    a, sa = _quantize(_silu(u[..., :f]) * u[..., f:])
    v = torch.matmul(a * sa, s["w2"].float().transpose(1, 2)) * s["s2"][:, None]
    full = torch.zeros(tk, c["experts"], device="cuda").scatter_(1, ids, p)
    return (v * full.t()[..., None]).sum(dim=0).to(s["out"].dtype)


_PLAIN = dict(norm=_norm, norm_grad=_norm_grad, gate=_gate, gate_grad=_gate_grad, product=_product, moe=_moe)


# ------------------------------------------------------------------------------------------------------------- calls
def _run_own(s):
    import paper_1609_07061_amd as q

    c = s["case"]
    kind = c["kind"]
    if kind == "norm":
        total = q.qnn_rms_norm_quant(s["x"], s["gamma"], _EPS, s.get("residual"), s["codes"], s["scale"], s.get("total"))[2]
        torch.mul(s["codes"], s["scale"][:, None], out=s["values"])
        return [s["values"], s["scale"]] + ([total] if c["residual"] else [])
    if kind == "norm_grad":
        return list(q.qnn_rms_norm_backward(s["grad"], s["x"], s["gamma"], _EPS, s.get("residual"), s["out"], s["gw"], s["ws"]))
    if kind == "gate":
        u, f = s["u"], c["width"]
        q.qnn_silu_gate_quant(u[:, :f], u[:, f:], s["codes"], s["scale"])
        torch.mul(s["codes"], s["scale"][:, None], out=s["values"])
        return [s["values"], s["scale"]]
    if kind == "gate_grad":
        u, o, f = s["u"], s["out"], c["width"]
        q.qnn_silu_gate_backward(s["grad"], u[:, :f], u[:, f:], o[:, :f], o[:, f:])
        return o
    if kind == "product":
        return q.qnn_int8_gemm(s["a"], s["sa"], s["w"], s["sw"], s.get("bias"), s["out"])
    return q.qnn_int8_moe(s["x"], s["sx"], s["logits"], c["top"], s["w1"], s["s1"], s["w2"], s["s2"], s["out"], s["ws"])


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state)


# -------------------------------------------------------------------------------------------------- cost, correctness
def work(case):
    """Inputs read once and outputs written once (codes: one byte), and the operations of the formulas; of the experts'
    weights those that the tokens choose, at most top of each token."""
    kind, w = case["kind"], _BYTES[case["type"]]
    if kind in ("norm", "norm_grad"):
        n, k = case["rows"] * case["width"], case["width"]
        more = 1 if case["residual"] else 0
        if kind == "norm":
            return dict(bytes=n * (w * (1 + 2 * more) + 1) + 4 * case["rows"] + w * k, flops=8 * n)
        return dict(bytes=n * w * (3 + more) + (w + 4) * k, flops=14 * n)
    if kind in ("gate", "gate_grad"):
        n = case["rows"] * case["width"]
        if kind == "gate":
            return dict(bytes=n * (2 * w + 1) + 4 * case["rows"], flops=8 * n)
        return dict(bytes=n * 5 * w, flops=12 * n)
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return dict(bytes=m * k + n * k + 4 * (m + n * (2 if case["bias"] else 1)) + m * n * w, flops=2 * m * n * k)
    tk, k, e, h, f = case["tokens"], case["top"], case["experts"], case["hidden"], case["inner"]
    chosen = e * (1 - (1 - k / e) ** tk)  # experts that some token chooses, on average
    return dict(bytes=int(chosen * (3 * f * h + 4 * (2 * f + h))) + tk * (h + 4 + 4 * e) + tk * h * w, flops=6 * tk * k * f * h)


def _exact_codes(y):
    top = y.abs().amax(dim=-1, keepdim=True)
    return torch.where(top > 0, torch.round(y * 127 / top), 0.0), top / 127


def exact(case, seed):
    d, kind = {k: v.double() for k, v in _inputs(case, seed).items()}, case["kind"]
    if kind in ("norm", "norm_grad"):
        extra = [d["residual"]] if case["residual"] else []
        h = d["x"] + extra[0] if extra and kind == "norm" else d["x"]
        rms = torch.sqrt(h.square().sum(dim=1, keepdim=True) / case["width"] + _EPS)
        if kind == "norm":
            q, s = _exact_codes(h / rms * d["gamma"])
            return [q * s, s[:, 0]] + ([h] if extra else [])
        unit = h / rms
        wg = d["grad"] * d["gamma"]
        gh = (wg - unit * (wg * unit).sum(dim=1, keepdim=True) / case["width"]) / rms
        return [gh + extra[0] if extra else gh, (d["grad"] * unit).sum(dim=0)]
    if kind in ("gate", "gate_grad"):
        a, b = d["u"].split(case["width"], dim=1)
        sig = torch.sigmoid(a)
        if kind == "gate":
            q, s = _exact_codes(a * sig * b)
            return [q * s, s[:, 0]]
        return torch.cat([d["grad"] * b * (sig + a * sig * torch.sigmoid(-a)), d["grad"] * a * sig], dim=1)
    if kind == "product":
        y = torch.mm(d["a"], d["w"].t()) * torch.outer(d["sa"], d["sw"])
        return y + d["bias"] if case["bias"] else y
    out = torch.zeros(case["tokens"], case["hidden"], dtype=torch.float64, device="cuda")
    for i, row in enumerate(d["logits"].tolist()):
        best = sorted(range(case["experts"]), key=lambda e: (-row[e], e))[:case["top"]]
        odds = [math.exp(row[e] - row[best[0]]) for e in best]
        for e, o in zip(best, odds):
            u = (d["w1"][e] @ d["x"][i]) * d["sx"][i] * d["s1"][e]
            a, b = u.split(case["inner"])
            q, s = _exact_codes(a * torch.sigmoid(a) * b)
            out[i] += (d["w2"][e] @ q) * s * d["s2"][e] * (o / sum(odds))
    return out
