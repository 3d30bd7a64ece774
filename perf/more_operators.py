"""Performance cases of the attention half of a decoder block on int8 codes: norm and position rotation of the heads of queries and keys with their
gradient, keys and values appended to a paged cache of codes, attention over that cache (single tokens, trees of drafted tokens, parts of prompts),
and rows to codes.

`own` False: every operator in its plain form, elementary torch operations in fp32 (angles in fp64); True: the package's entry points.

Cached keys and values are int8 codes with one fp32 scale for each token and head.  Outputs that are held as codes are returned as the values they stand
for, code * scale in bfloat16, with the scales beside them.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_EPS = 1e-6


# ------------------------------------------------------------------------------------------------------------- cases
def _rotate(kind, tokens, heads, kv, size, type, axes=1, pairs=None, neighbours=False, norm=True):
    return dict(kind=kind, tokens=tokens, heads=heads, kv=kv, size=size, type=type, axes=axes, pairs=size // 2 if pairs is None else pairs,
                neighbours=neighbours, norm=norm)


def _append(sequences, new, longest, heads, kv, size, type, page, norm=True):
    return dict(kind="append", sequences=sequences, new=new, longest=longest, heads=heads, kv=kv, size=size, type=type, axes=1, pairs=size // 2,
                neighbours=False, norm=norm, page=page)


def _attend(sequences, new, longest, heads, kv, size, type, page, cap=0.0, slopes=False, tree=False):
    return dict(kind="attend", sequences=sequences, new=new, longest=longest, heads=heads, kv=kv, size=size, type=type, page=page, cap=cap, slopes=slopes,
                tree=tree)


def listed():
    return [
        # A serving batch of 20 tokens: heads of queries and keys normed and rotated, three axes of positions (image and video tokens).
        dict(name="rotate_batch", **_rotate("rotate", 20, 32, 8, 128, "bf16", axes=3)),
        # A training window of 8192 tokens.
        dict(name="rotate_8192", **_rotate("rotate", 8192, 32, 8, 128, "bf16")),
        # Its gradient.
        dict(name="rotate_grad_8192", **_rotate("rotate_grad", 8192, 32, 8, 128, "bf16")),
        # Full precision, ragged batch, heads of 80 of which 64 are rotated, neighbouring pairs, three axes.
        dict(name="rotate_grad_odd", **_rotate("rotate_grad", 1999, 10, 5, 80, "f32", axes=3, pairs=32, neighbours=True)),
        # One new token for each of 64 sequences of a serving step.
        dict(name="append_batch", **_append(64, 1, 200, 32, 8, 128, "bf16", 16)),
        # A prompt of 4096 tokens into the cache.
        dict(name="append_prompt", **_append(1, 4096, 4096, 32, 8, 128, "bf16", 64)),
        # One token of one long sequence: latency.
        dict(name="attend_token", **_attend(1, 1, 10000, 32, 8, 128, "bf16", 16)),
        # A serving step of 64 sequences of up to 8192 tokens.
        dict(name="attend_batch", **_attend(64, 1, 8192, 32, 8, 128, "bf16", 64)),
        # Trees of 40 drafted tokens to be checked in 8 sequences, capped scores.
        dict(name="attend_tree", **_attend(8, 40, 4099, 16, 4, 128, "f16", 16, cap=50.0, tree=True)),
        # The last 2048 tokens of a prompt of 8192, scores with a bias by distance.
        dict(name="attend_prompt", **_attend(1, 2048, 8192, 32, 8, 128, "bf16", 64, slopes=True)),
        # The attention's result to codes in front of the output product, one token.
        dict(name="quant_token", kind="quant", rows=1, width=4096, type="bf16"),
        # The same for a prompt.
        dict(name="quant_8192", kind="quant", rows=8192, width=4096, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate_grad", "append", "append", "attend", "attend", "attend", "attend", "quant"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "quant":
        return dict(kind=kind, rows=_log_int(rng, 1, 8192), width=_log_int(rng, 64, 4096), type=t)
    kv, group, size = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 64, 80, 112, 128, 128, 128, 256])
    heads = kv * group
    if kind in ("rotate", "rotate_grad"):
        pairs = size // 2 if rng.random() < 0.7 else size // 32 * 8
        return _rotate(kind, _log_int(rng, 1, max(1, 8192 * 40 * 128 // (size * (heads + kv)) // 2)), heads, kv, size, t, rng.choice([1, 1, 3]), pairs,
                       rng.random() < 0.3, rng.random() < 0.8)
    page = rng.choice([16, 16, 32, 64, 20, 128])
    if kind == "append":
        sequences = _log_int(rng, 1, 64)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, 4096 * 48 * 128 // (size * (heads + 2 * kv)) // 2 // sequences))
        return _append(sequences, new, new + rng.randint(0, 200), heads, kv, size, t, page, rng.random() < 0.7)
    mode = rng.choice(["token", "token", "tree", "prompt"])
    cap, slopes = (rng.choice([20.0, 50.0]) if rng.random() < 0.3 else 0.0), rng.random() < 0.25
    if mode == "token":
        sequences = _log_int(rng, 1, 64)
        return _attend(sequences, 1, _log_int(rng, 1, min(32768, 1 << 18 >> (sequences.bit_length() - 1))), heads, kv, size, t, page, cap, slopes)
    if mode == "tree":
        new, sequences = rng.randint(2, 64), _log_int(rng, 1, 16)
        return _attend(sequences, new, new + _log_int(rng, 1, 4096), heads, kv, size, t, page, cap, slopes, True)
    sequences, new = rng.choice([1, 1, 2, 3]), _log_int(rng, 65, 1024)
    return _attend(sequences, new, new + _log_int(rng, 1, 3000), heads, kv, size, t, page, cap, slopes)


# ------------------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """(lengths, new tokens) of the sequences: the first is the longest, the others spread over the upper nine tenths; where there are many new tokens, they
    are fewer in every other sequence."""
    n, new, longest = case["sequences"], case["new"], case["longest"]
    lengths, news = [], []
    for b in range(n):
        fresh = new if b % 2 == 0 or case.get("tree") else (new + 1) // 2
        spread = (b * 37 % n) / n
        news.append(fresh)
        lengths.append(max(fresh, longest - int(0.9 * spread * longest)))
    return lengths, news


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, device="cuda", dtype=dtype)


def _rotation(case, d, g, first=None):
    """Positions, frequencies and the axis of every pair; first: the positions' beginnings are given, token by token."""
    pairs, axes, t = case["pairs"], case["axes"], d["tokens"]
    d["freq"] = (10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs))
    if first is not None:
        d["positions"] = first[None]
    elif axes == 1:  # far into a document
        d["positions"] = torch.arange(t, device="cuda", dtype=torch.int32)[None] + torch.randint(0, 200000, (1, 1), generator=g, device="cuda", dtype=torch.int32)
    else:  # time, height and width
        d["positions"] = torch.stack([torch.randint(0, m, (t,), generator=g, device="cuda", dtype=torch.int32) for m in (100000, 64, 64)])
    d["axis"] = None if axes == 1 else torch.arange(pairs, device="cuda", dtype=torch.int32) * axes // pairs


def _heads(case, t, d, g, values):
    """Queries, keys (and values) as one product leaves them side by side, and the norms' weights."""
    heads, kv, size = case["heads"], case["kv"], case["size"]
    n = heads + (2 if values else 1) * kv
    rows = (_normal(g, d["tokens"], n, size) * torch.exp(0.5 * _normal(g, n, size))).to(t)
    d["q"], d["k"] = rows[:, :heads], rows[:, heads:heads + kv]
    if values:
        d["v"] = rows[:, heads + kv:]
    d["gamma_q"] = (1 + 0.1 * _normal(g, size)).to(t) if case["norm"] else None
    d["gamma_k"] = (1 + 0.1 * _normal(g, size)).to(t) if case["norm"] else None


def _pages(case, d, g):
    """A cache with pages in any order, and the sequences' tables; entries that no sequence needs hold -1."""
    lengths, news = _lengths(case)
    page, kv, size = case["page"], case["kv"], case["size"]
    need = [-(-n // page) for n in lengths]
    total = sum(need) + 3
    order = torch.randperm(total, generator=g, device="cuda")[:sum(need)].to(torch.int32)
    table = torch.full((len(need), max(need)), -1, device="cuda", dtype=torch.int32)
    rows = torch.repeat_interleave(torch.arange(len(need), device="cuda"), _ints(need, torch.int64))
    at = torch.cat([torch.arange(n, device="cuda") for n in need])
    table[rows, at] = order
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    codes = lambda: _normal(g, total, kv, page, size).mul_(32).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
    scale = lambda: torch.rand(total, kv, page, generator=g, device="cuda") * 0.03 + 0.01  # noqa: E731
    d["cache"] = (codes(), scale(), codes(), scale())
    d.update(table=table, starts=_ints(starts), lengths=_ints(lengths), tokens=starts[-1])
    # where a token is: its sequence, and its index there
    d["sequence"] = torch.repeat_interleave(torch.arange(len(news), device="cuda"), _ints(news, torch.int64))
    d["index"] = torch.cat([torch.arange(n - k, n, device="cuda") for n, k in zip(lengths, news)])


def _trees(case, seed):
    """Masks of drafted tokens: a token sees itself and those that it follows.  Branches are short, most tokens follow the one before."""
    rng, out = random.Random(seed), []
    for n in _lengths(case)[1]:
        masks = []
        for i in range(n):
            parent = i - 1 if rng.random() < 0.6 else rng.randint(-1, i - 1)
            masks.append((masks[parent] if parent >= 0 else 0) | 1 << i)
        out += masks
    return _ints([m - (1 << 64) if m >> 63 else m for m in out], torch.int64)


def _inputs(case, seed):
    """Inputs of a case, on the GPU, from the seed alone."""
    g, kind, t, d = _gen(seed), case["kind"], _TYPES[case["type"]], {}
    if kind == "quant":
        d["x"] = _normal(g, case["rows"], case["width"]).to(t)
    elif kind in ("rotate", "rotate_grad"):
        d["tokens"] = case["tokens"]
        _heads(case, t, d, g, False)
        _rotation(case, d, g)
        if kind == "rotate_grad":
            d["grad_q"] = (0.1 * _normal(g, case["tokens"], case["heads"], case["size"])).to(t)
            d["grad_k"] = (0.1 * _normal(g, case["tokens"], case["kv"], case["size"])).to(t)
    else:
        _pages(case, d, g)
        if kind == "append":
            _heads(case, t, d, g, True)
            _rotation(case, d, g, d["index"].to(torch.int32))
        else:
            d["q"] = (2 * _normal(g, d["tokens"], case["heads"], case["size"])).to(t)
            d["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case["heads"] + 1, device="cuda", dtype=torch.float32) / case["heads"]) if case["slopes"] else None
            d["tree"] = _trees(case, seed) if case["tree"] else None
    return d


def prepare(case, seed):
    """Inputs, cache, tables, and the outputs and workspaces that a program keeps between calls."""
    d, kind, t = _inputs(case, seed), case["kind"], _TYPES[case["type"]]
    new = lambda *shape, dtype=t: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    st = dict(case=case, **d)
    if kind == "quant":
        r, w = case["rows"], case["width"]
        st.update(codes=new(r, w, dtype=torch.int8), scale=new(r, dtype=torch.float32), values=new(r, w, dtype=torch.bfloat16))
        return st
    st["out"] = torch.empty_like(st["q"], memory_format=torch.contiguous_format)
    if kind in ("rotate", "rotate_grad"):
        st["out_k"] = torch.empty_like(st["k"], memory_format=torch.contiguous_format)
    if kind == "rotate_grad" and case["norm"]:
        st.update(gq=new(case["size"], dtype=torch.float32), gk=new(case["size"], dtype=torch.float32))
    if kind == "append":
        st["values"] = [torch.empty_like(st["cache"][i], dtype=torch.bfloat16) for i in (0, 2)]
    if kind == "attend":
        # (for the plain form: the row of a padded batch that every token is, and back)
        news = _lengths(case)[1]
        most = max(news)
        st["flat"] = torch.cat([b * most + torch.arange(n, device="cuda") for b, n in enumerate(news)])
        st["padded"] = torch.stack([torch.clamp(torch.arange(most, device="cuda"), max=n - 1) for n in news]) + st["starts"][:-1, None]
    if own:
        import paper_1609_07061_amd as q

        need = 0
        if kind == "rotate_grad":
            need = q.qnn_qk_norm_rotate_backward_workspace_bytes(d["tokens"], case["heads"], case["kv"], case["size"])
        elif kind == "attend":
            need = q.qnn_cache_attention_workspace_bytes(d["tokens"], case["sequences"], case["heads"], case["kv"], case["size"], case["new"], case["longest"])
        st["workspace"] = new(max(need, 1), dtype=torch.uint8)
    return st


# ------------------------------------------------------------------------------------------------------- plain forms
def _quantize(y):
    """(codes as fp32, scales) of every row."""
    scale = y.abs().amax(dim=-1, keepdim=True) / 127
    return torch.where(scale > 0, torch.round(y / scale), 0.0), scale[..., 0]


def _angles(s):
    """Cosine and sine [tokens][1][pairs] in fp32 of angles in fp64."""
    p = s["positions"].double()
    at = p[0][:, None] if s["axis"] is None else p[s["axis"].long()].t()
    a = at * s["freq"]
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _turn(y, cos, sin, neighbours):
    pairs = cos.shape[-1]
    a, b = (y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]) if neighbours else (y[..., :pairs], y[..., pairs:2 * pairs])
    u, v = a * cos - b * sin, b * cos + a * sin
    both = torch.stack([u, v], dim=-1).flatten(-2) if neighbours else torch.cat([u, v], dim=-1)
    return torch.cat([both, y[..., 2 * pairs:]], dim=-1)


def _factor(h):
    return torch.rsqrt((h * h).mean(dim=-1, keepdim=True) + _EPS)


def _normed_turned(x, gamma, cos, sin, neighbours):
    h = x.float()
    if gamma is not None:
        h = h * _factor(h) * gamma.float()
    return _turn(h, cos, sin, neighbours)


def _rotate_plain(s):
    cos, sin = _angles(s)
    n, t = s["case"]["neighbours"], s["q"].dtype
    return [_normed_turned(s[x], s["gamma_" + x], cos, sin, n).to(t) for x in ("q", "k")]


def _rotate_grad_plain(s):
    cos, sin = _angles(s)
    n, t = s["case"]["neighbours"], s["q"].dtype
    out, weights = [], []
    for x in ("q", "k"):
        g = _turn(s["grad_" + x].float(), cos, -sin, n)
        if s["gamma_" + x] is not None:
            h = s[x].float()
            r = _factor(h)
            wg = g * s["gamma_" + x].float()
            weights.append((g * h * r).sum(dim=(0, 1)))
            g = r * (wg - h * (r * r) * (wg * h).mean(dim=-1, keepdim=True))
        out.append(g.to(t))
    return out + weights


def _append_plain(s):
    cos, sin = _angles(s)
    page = s["case"]["page"]
    pages = s["table"][s["sequence"], s["index"] // page].long()
    off = s["index"] % page
    for i, y in ((0, _normed_turned(s["k"], s["gamma_k"], cos, sin, False)), (2, s["v"].float())):
        codes, scale = _quantize(y)
        s["cache"][i][pages, :, off] = codes.to(torch.int8)
        s["cache"][i + 1][pages, :, off] = scale
    return _cache_values(s) + [_normed_turned(s["q"], s["gamma_q"], cos, sin, False).to(s["q"].dtype)]


def _cache_values(s):
    out = []
    for i, values in zip((0, 2), s["values"]):
        torch.mul(s["cache"][i], s["cache"][i + 1][..., None], out=values)
        out += [values, s["cache"][i + 1]]
    return out


def _attend_plain(s):
    c = s["case"]
    n, kv, group, size, page, longest = c["sequences"], c["kv"], c["heads"] // c["kv"], c["size"], c["page"], c["longest"]
    longest = max(longest, c["new"])
    table = s["table"].clamp(min=0).long()

    def whole(codes, scale):
        x = codes[table].float() * scale[table][..., None]  # [sequence][page][kv][token][size]
        return x.transpose(1, 2).reshape(n, kv, -1, size)[:, :, :longest].contiguous()

    rows = s["padded"]
    most = rows.shape[1]
    q = s["q"][rows].float().view(n, most, kv, group, size).permute(0, 2, 3, 1, 4).reshape(n, kv, group * most, size)
    x = torch.matmul(q, whole(*s["cache"][:2]).transpose(2, 3)).mul_(1 / math.sqrt(size))
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    x = x.view(n, kv, group, most, longest)
    lengths, key = s["lengths"][:, None], torch.arange(longest, device="cuda")
    base = lengths - (s["starts"][1:] - s["starts"][:-1])[:, None]
    if c["tree"]:
        bits = s["tree"][rows]  # [sequence][query]
        drafted = key[None, None] - base[..., None]  # [sequence][1][key]
        seen = (drafted < 0) | ((drafted < 64) & ((bits[..., None] >> drafted.clamp(0, 63)) & 1).bool())
        seen &= key < lengths[..., None]
    else:
        at = base + torch.arange(most, device="cuda")
        seen = key <= torch.minimum(at, lengths - 1)[..., None]
    if s["slopes"] is not None:
        if c["tree"]:
            ones = ((s["tree"][:, None] >> torch.arange(64, device="cuda")) & 1).sum(dim=1)  # of every drafted token: its depth
            at = base + ones[rows] - 1
            depth = ones[rows].gather(1, (key[None] - base).clamp(0, most - 1))
            from_ = torch.where(key[None] < base, key[None], base + depth - 1)
        else:
            from_ = key[None]
        x = x - s["slopes"].view(kv, group, 1, 1) * (at[:, :, None] - from_[:, None]).float()[:, None, None]
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True).clamp_(min=-1e30)
    x = torch.exp(x - top)
    total = x.sum(dim=-1, keepdim=True)
    y = torch.matmul(x.view(n, kv, group * most, longest), whole(*s["cache"][2:])).view(n, kv, group, most, size)
    y = torch.where(total > 0, y / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n * most, c["heads"], size)
    return y[s["flat"]].to(s["q"].dtype)


def _quant_plain(s):
    codes, scale = _quantize(s["x"].float())
    return [(codes * scale[:, None]).to(torch.bfloat16), scale]


_PLAIN = dict(rotate=_rotate_plain, rotate_grad=_rotate_grad_plain, append=_append_plain, attend=_attend_plain, quant=_quant_plain)


# ------------------------------------------------------------------------------------------------------------- calls
def _run_own(s):
    import paper_1609_07061_amd as q

    c = s["case"]
    kind = c["kind"]
    if kind == "rotate":
        return list(q.qnn_qk_norm_rotate(s["q"], s["k"], s["gamma_q"], s["gamma_k"], _EPS, s["positions"], s["freq"], s["axis"], c["neighbours"], s["out"],
                                         s["out_k"]))
    if kind == "rotate_grad":
        got = q.qnn_qk_norm_rotate_backward(s["grad_q"], s["grad_k"], s["q"], s["k"], s["gamma_q"], s["gamma_k"], _EPS, s["positions"], s["freq"], s["axis"],
                                            c["neighbours"], s["out"], s["out_k"], s.get("gq"), s.get("gk"), s["workspace"])
        return [x for x in got if x is not None]
    if kind == "append":
        out = q.qnn_cache_append(s["cache"], s["table"], s["starts"], s["lengths"], s["k"], s["v"], s["gamma_k"], _EPS, s["positions"], s["freq"], s["axis"],
                                 c["neighbours"], s["q"], s["gamma_q"], s["out"])
        return _cache_values(s) + [out]
    if kind == "attend":
        return q.qnn_cache_attention(s["q"], s["cache"], s["table"], s["starts"], s["lengths"], 1 / math.sqrt(c["size"]), c["cap"], s["slopes"], s["tree"],
                                     c["new"], c["longest"], s["out"], s["workspace"])
    q.qnn_rows_quant(s["x"], s["codes"], s["scale"])
    torch.mul(s["codes"], s["scale"][:, None], out=s["values"])
    return [s["values"], s["scale"]]


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state)


# -------------------------------------------------------------------------------------------------- cost, correctness
def work(case):
    """Inputs read once and outputs written once (codes: one byte, and the cached tokens of the sequences, not spare pages), and the operations of the
    formulas."""
    kind, w = case["kind"], _BYTES[case["type"]]
    if kind == "quant":
        n = case["rows"] * case["width"]
        return dict(bytes=n * (w + 1) + 4 * case["rows"], flops=4 * n)
    heads, kv, size = case["heads"], case["kv"], case["size"]
    if kind in ("rotate", "rotate_grad"):
        n = case["tokens"] * (heads + kv) * size
        more = 4 * case["tokens"] * case["axes"] + 8 * case["pairs"]
        return dict(bytes=n * w * (3 if kind == "rotate_grad" else 2) + more, flops=n * (16 if kind == "rotate_grad" else 8))
    lengths, news = _lengths(case)
    tokens = sum(news)
    if kind == "append":
        return dict(bytes=tokens * (2 * heads * size * w + 2 * kv * (size * (w + 1) + 4)), flops=tokens * (heads + 2 * kv) * size * 8)
    pairs = sum(k * (n - k) + k * (k + 1) // 2 for n, k in zip(lengths, news))
    return dict(bytes=2 * tokens * heads * size * w + sum(lengths) * 2 * kv * (size + 4), flops=4 * size * heads * pairs)


def _exact_codes(y):
    top = y.abs().amax(dim=-1, keepdim=True)
    return torch.where(top > 0, torch.round(y * 127 / torch.where(top > 0, top, 1.0)), 0.0), top / 127


def _exact_turn(y, d, case, sign):
    """The pairs as complex numbers, turned."""
    pairs = case["pairs"]
    at = d["positions"].double()[0].unsqueeze(1).expand(-1, pairs) if d["axis"] is None else d["positions"].double().index_select(0, d["axis"]).t()
    unit = torch.polar(torch.ones_like(at), sign * at * d["freq"]).unsqueeze(1)
    out = y.clone()
    if case["neighbours"]:
        z = torch.complex(y[..., 0:2 * pairs:2].contiguous(), y[..., 1:2 * pairs:2].contiguous()) * unit
        out[..., 0:2 * pairs:2], out[..., 1:2 * pairs:2] = z.real, z.imag
    else:
        z = torch.complex(y[..., :pairs].contiguous(), y[..., pairs:2 * pairs].contiguous()) * unit
        out[..., :pairs], out[..., pairs:2 * pairs] = z.real, z.imag
    return out


def _exact_heads(d, case, name):
    x = d[name].double()
    if case["norm"]:
        x = x / torch.sqrt(x.square().sum(dim=2, keepdim=True) / case["size"] + _EPS) * d["gamma_" + name].double()
    return _exact_turn(x, d, case, 1.0)


def _exact_grad(d, case, name):
    g = _exact_turn(d["grad_" + name].double(), d, case, -1.0)
    if not case["norm"]:
        return g, None
    x = d[name].double()
    rms = torch.sqrt(x.square().sum(dim=2, keepdim=True) / case["size"] + _EPS)
    unit = x / rms
    wg = g * d["gamma_" + name].double()
    return (wg - unit * (wg * unit).sum(dim=2, keepdim=True) / case["size"]) / rms, (g * unit).sum(dim=1).sum(dim=0)


def _exact_attend(d, case):
    """Sequence by sequence and head by head."""
    lengths, news = _lengths(case)
    kv, size, page = case["kv"], case["size"], case["page"]
    group, out, first = case["heads"] // kv, torch.zeros(d["q"].shape, dtype=torch.float64, device="cuda"), 0
    codes_k, scale_k, codes_v, scale_v = d["cache"]
    trees = d["tree"].tolist() if case["tree"] else None
    for b, (n, k) in enumerate(zip(lengths, news)):
        at = torch.arange(n, device="cuda")
        pages, off = d["table"][b].long()[at // page], at % page
        query = torch.arange(n - k, n, device="cuda")
        sees, where, from_ = at[None, :] <= query[:, None], query, at
        if trees:
            rows = [[(m >> i) & 1 for i in range(k)] for m in trees[first:first + k]]
            sees = torch.cat([torch.ones(k, n - k, device="cuda", dtype=torch.bool), _ints(rows).bool()], dim=1)
            where = n - k - 1 + _ints([sum((m >> i) & 1 for i in range(64)) for m in trees[first:first + k]])
            from_ = torch.cat([at[:n - k], where])
        for h in range(kv):
            key = codes_k[pages, h, off].double() * scale_k[pages, h, off].double()[:, None]
            value = codes_v[pages, h, off].double() * scale_v[pages, h, off].double()[:, None]
            for j in range(h * group, (h + 1) * group):
                x = (d["q"][first:first + k, j].double() @ key.t()) / math.sqrt(size)
                if case["cap"]:
                    x = torch.tanh(x / case["cap"]) * case["cap"]
                if d["slopes"] is not None:
                    x = x + d["slopes"][j].double() * (from_[None, :] - where[:, None])
                p = torch.softmax(torch.where(sees, x, -math.inf), dim=1)
                out[first:first + k, j] = torch.where(sees.any(dim=1, keepdim=True), p @ value, 0.0)
        first += k
    return out


def exact(case, seed):
    d, kind = _inputs(case, seed), case["kind"]
    if kind == "quant":
        codes, scale = _exact_codes(d["x"].double())
        return [codes * scale, scale[:, 0]]
    if kind == "rotate":
        return [_exact_heads(d, case, "q"), _exact_heads(d, case, "k")]
    if kind == "rotate_grad":
        (gq, wq), (gk, wk) = _exact_grad(d, case, "q"), _exact_grad(d, case, "k")
        return [gq, gk] + ([wq, wk] if case["norm"] else [])
    if kind == "attend":
        return _exact_attend(d, case)
    out, at = [], d["index"]
    where = (d["table"].long()[d["sequence"], torch.div(at, case["page"], rounding_mode="floor")], torch.remainder(at, case["page"]))
    for i, y in ((0, _exact_heads(d, case, "k")), (2, d["v"].double())):
        codes, scales = d["cache"][i].double(), d["cache"][i + 1].double()
        c, s = _exact_codes(y)
        for h in range(case["kv"]):
            codes[where[0], h, where[1]], scales[where[0], h, where[1]] = c[:, h], s[:, h, 0]
        out += [codes * scales[..., None], scales]
    return out + [_exact_heads(d, case, "q")]
