"""The operators around the sparse attention of a transformer layer, as a list of measurable cases.

Kinds (`op`):
  table        cosines and sines of the rotary angles of a token grid, for one to three axes, scaled for long contexts or not
  rope         per-head RMS norm of queries and keys with the position rotation in the same pass (`norm` False: the rotation
               alone; `rot` 0: the norm alone)
  rope_grad    its gradients, with respect to queries, keys and the two norm weights
  cross        attention of a layer's tokens to another sequence's keys and values (an encoder's states), with a length of its
               own for every entry of the batch and key heads shared by groups of query heads
  cross_grad   its gradients, with respect to queries, keys and values
Tensors are [B, H, L, d] by shape; `storage` says how they lie in memory.

`own` False computes an operator in its plain form, True by the calls of `paper_2509_16518_amd.fgattn`.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_EPS = 1e-6


def _table(sizes, pairs, theta=10000.0, factor=1.0, original=0.0, mscale=1.0):
    return {"op": "table", "sizes": "x".join(map(str, sizes)), "pairs": "x".join(map(str, pairs)), "theta": theta, "factor": factor,
            "original": original, "mscale": mscale}


def _rope(op, B, Hq, Hk, L, d, rot, layout="interleaved", dtype="bf16", norm=True, positions=False, storage="bhld"):
    return {"op": op, "B": B, "Hq": Hq, "Hk": Hk, "L": L, "d": d, "rot": rot, "layout": layout, "dtype": dtype, "norm": norm,
            "positions": positions, "storage": storage}


def _cross(op, B, Hkv, group, Lq, Lk, d, ragged=False, storage="bhld"):
    return {"op": op, "B": B, "Hkv": Hkv, "group": group, "Lq": Lq, "Lk": Lk, "d": d, "ragged": ragged, "storage": storage}


def listed():
    named = {
        # the angles of the Wan shape's token grid (time, height, width), once per resolution
        "table-wan-grid": _table((21, 30, 52), (22, 21, 21)),
        # one long axis, scaled to eight times the trained length by wavelength
        "table-long-scaled": _table((118800,), (64,), theta=1e6, factor=8.0, original=16384.0, mscale=1.2079),
        # one new token of each of eight sequences at its own position: launches and latency count
        "rope-token": _rope("rope", 8, 12, 12, 1, 128, 128, positions=True),
        # queries and keys of a short clip in a small model: batch of two, tokens-first storage, part of the head in halves, fp16
        "rope-clip-half": _rope("rope", 2, 8, 8, 2635, 64, 48, layout="half", dtype="fp16", storage="blhd"),
        # queries and keys of one layer of the HunyuanVideo shape, as the projection leaves them
        "rope-hunyuan": _rope("rope", 1, 24, 24, 118800, 128, 128, storage="blhd"),
        # a training step of the same small model
        "rope-grad-clip-half": _rope("rope_grad", 2, 8, 8, 2635, 64, 48, layout="half", dtype="fp16", storage="blhd"),
        # a training step of the Wan-2.1-1.3B shape
        "rope-grad-wan": _rope("rope_grad", 1, 12, 12, 32760, 128, 128),
        # one token of each of four sequences against long encoder states of odd lengths, five query heads to a key head
        "cross-token": _cross("cross", 4, 8, 5, 1, 8191, 128, ragged=True),
        # a layer of the Wan shape over the states of a padded text
        "cross-wan": _cross("cross", 1, 12, 1, 32760, 512, 128),
        # a layer of the HunyuanVideo shape over a shorter text, tokens-first storage (the largest forward call)
        "cross-hunyuan": _cross("cross", 1, 24, 1, 118800, 256, 128, storage="blhd"),
        # a training step of the small model: texts of odd lengths
        "cross-grad-clip": _cross("cross_grad", 2, 8, 1, 2635, 77, 64, ragged=True, storage="blhd"),
        # a training step of the Wan shape
        "cross-grad-wan": _cross("cross_grad", 1, 12, 1, 32760, 512, 128),
    }
    return [dict(case, name=name) for name, case in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(("table", "rope", "rope_grad", "cross", "cross_grad"), (2, 4, 3, 5, 4))[0]
    while True:
        if op == "table":
            axes = rng.randint(1, 3)
            sizes = [_log(rng, 1, 118800)] if axes == 1 else [rng.randint(1, 40)] + [_log(rng, 2, 90) for _ in range(axes - 1)]
            pairs = [rng.randint(4, 64 // axes) for _ in range(axes)]
            scaled = rng.random() < 0.5
            case = _table(sizes, pairs, theta=rng.choice((256.0, 10000.0, 500000.0)), factor=rng.uniform(1.5, 32.0) if scaled else 1.0,
                          original=rng.choice((0.0, 4096.0, 32768.0)) if scaled else 0.0, mscale=rng.choice((1.0, 1.1, 1.25)))
            if math.prod(sizes) <= 118800:
                return case
        elif op in ("rope", "rope_grad"):
            d = rng.choice((64, 128, 128, 96, 256))
            Hk = _log(rng, 1, 40)
            case = _rope(op, rng.choice((1, 1, 2, 4)), Hk * rng.choice((1, 1, 1, 2, 4)), Hk, _log(rng, 1, 118800), d,
                         rng.choice((d, d, d // 2, 3 * d // 8 // 2 * 2, 0)), layout=rng.choice(("interleaved", "half")),
                         dtype=rng.choice(("bf16", "bf16", "fp16", "fp32")), norm=rng.random() < 0.75, positions=rng.random() < 0.3,
                         storage=rng.choice(("bhld", "blhd")))
            if not case["norm"] and not case["rot"]:
                case["norm"] = True
            limit = work(listed()[4]) if op == "rope" else work(listed()[6])
            if case["Hq"] <= 40 and work(case)["bytes"] <= limit["bytes"]:
                return case
        else:
            Hkv = _log(rng, 1, 40)
            case = _cross(op, rng.choice((1, 1, 2, 4)), Hkv, rng.choice((1, 1, 1, 2, 5, 8)), _log(rng, 1, 118800), _log(rng, 1, 8192),
                          rng.choice((64, 128, 128)), ragged=rng.random() < 0.5, storage=rng.choice(("bhld", "blhd")))
            limit = 24 * 118800 * 256 if op == "cross" else 12 * 32760 * 512
            if Hkv * case["group"] <= 40 and case["B"] * Hkv * case["group"] * case["Lq"] * case["Lk"] <= limit:
                return case


def _ints(text):
    return [int(x) for x in text.split("x")]


def _key_lengths(c):
    """How many keys each entry of the batch has: the first one all, the others shorter."""
    return [c["Lk"] if b == 0 or not c["ragged"] else int(c["Lk"] * (0.6180339887 * b % 1.0)) for b in range(c["B"])]


def work(c):
    if c["op"] == "table":
        n = math.prod(_ints(c["sizes"])) * sum(_ints(c["pairs"]))
        return {"bytes": 8 * n, "flops": 4 * n}
    if c["op"] in ("rope", "rope_grad"):
        size = 4 if c["dtype"] == "fp32" else 2
        n = c["B"] * (c["Hq"] + c["Hk"]) * c["L"] * c["d"]
        tables = 4 * c["rot"] * c["L"] * (c["B"] if c["positions"] else 1)
        if c["op"] == "rope":
            return {"bytes": 2 * n * size + tables, "flops": n * ((4 if c["norm"] else 0) + 3)}
        return {"bytes": (3 if c["norm"] else 2) * n * size + tables, "flops": n * ((12 if c["norm"] else 0) + 3)}
    H, keys = c["Hkv"] * c["group"], sum(_key_lengths(c))
    rows, states = c["B"] * H * c["Lq"], c["Hkv"] * keys
    if c["op"] == "cross":
        return {"bytes": 4 * rows * c["d"] + 4 * rows + 4 * states * c["d"], "flops": 4 * c["d"] * H * c["Lq"] * keys}
    return {"bytes": 8 * rows * c["d"] + 4 * rows + 8 * states * c["d"], "flops": 10 * c["d"] * H * c["Lq"] * keys}


def _stored(c, data):
    """The values of `data` ([B, H, L, d]) in the case's storage order, seen as [B, H, L, d]."""
    return data.transpose(1, 2).contiguous().transpose(1, 2) if c["storage"] == "blhd" else data


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] == "table":
        # (size, pairs, theta, offset, step, factor, original, beta_fast, beta_slow) of each axis: the positions begin where an
        # earlier piece of the sequence ended
        begin = torch.randint(0, 2000, (3,), generator=gen, device="cuda").tolist()
        axes = [(n, m, c["theta"], float(begin[a]), 1.0, c["factor"], c["original"], 32.0, 1.0)
                for a, (n, m) in enumerate(zip(_ints(c["sizes"]), _ints(c["pairs"])))]
        return {"case": c, "axes": axes, "rows": math.prod(_ints(c["sizes"])), "pairs": sum(_ints(c["pairs"]))}
    if c["op"] in ("rope", "rope_grad"):
        def normal(H, gain):
            return _stored(c, (gain * torch.randn((c["B"], H, c["L"], c["d"]), generator=gen, device="cuda")).to(_TYPES[c["dtype"]]))
        s = {"case": c, "q": normal(c["Hq"], 2.0), "k": normal(c["Hk"], 0.5), "cos": None, "sin": None, "positions": None, "qw": None, "kw": None}
        if c["norm"]:
            s["qw"], s["kw"] = ((1.0 + 0.3 * torch.randn((c["d"],), generator=gen, device="cuda")).to(_TYPES[c["dtype"]]) for _ in "qk")
        if c["rot"]:
            rows = 2 * c["L"] + 15 if c["positions"] else c["L"]
            freq = 10000.0 ** (-torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) / (c["rot"] // 2))
            angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * freq
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
            if c["positions"]:
                s["positions"] = torch.randint(0, rows, (c["B"], c["L"]), generator=gen, device="cuda", dtype=torch.int32)
        if c["op"] == "rope_grad":
            s["dq_out"], s["dk_out"] = normal(c["Hq"], 0.02), normal(c["Hk"], 0.02)
        return s
    H = c["Hkv"] * c["group"]

    def normal(heads, L, gain=1.0):
        return _stored(c, (gain * torch.randn((c["B"], heads, L, c["d"]), generator=gen, device="cuda")).bfloat16())
    s = {"case": c, "q": normal(H, c["Lq"], 1.5), "k": normal(c["Hkv"], c["Lk"]), "v": normal(c["Hkv"], c["Lk"]), "scale": c["d"] ** -0.5,
         "k_lens": torch.tensor(_key_lengths(c), device="cuda", dtype=torch.int32) if c["ragged"] else None}
    if c["op"] == "cross_grad":
        out, s["lse"] = _plain_cross(s)
        s["out"] = _stored(c, out)
        s["dout"] = normal(H, c["Lq"], 0.02)
    return s


def _plain_table(s):
    parts, inner = [], s["rows"]
    row = torch.arange(s["rows"], device="cuda")
    for size, pairs, theta, offset, step, factor, original, fast, slow in s["axes"]:
        inner //= size
        freq = theta ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
        kept = ((original * freq / (2 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
        freq = freq * (kept + (1.0 - kept) / factor)
        parts.append((offset + step * ((row // inner) % size).double())[:, None] * freq)
    angle = torch.cat(parts, 1)
    return (angle.cos() * s["case"]["mscale"]).float(), (angle.sin() * s["case"]["mscale"]).float()


def _rotated(x, s, sign):
    """x (fp32) with the first `rot` elements of each row turned by the angle of its position (sign -1: turned back)."""
    rot = s["case"]["rot"]
    if not rot:
        return x
    if s["positions"] is not None:
        cos, sin = s["cos"][s["positions"].long()][:, None], sign * s["sin"][s["positions"].long()][:, None]
    else:
        cos, sin = s["cos"], sign * s["sin"]
    y = x.clone()
    if s["case"]["layout"] == "interleaved":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2] = a * cos - b * sin
        y[..., 1:rot:2] = a * sin + b * cos
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2] = a * cos - b * sin
        y[..., rot // 2:rot] = a * sin + b * cos
    return y


def _plain_rope(x, weight, s):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + _EPS) * weight.float()
    return _rotated(y, s, 1.0).to(x.dtype)


def _plain_rope_grad(x, weight, dy, s):
    dz = _rotated(dy.float(), s, -1.0)
    if weight is None:
        return dz.to(x.dtype), None
    rstd = torch.rsqrt(x.float().square().mean(-1, keepdim=True) + _EPS)
    unit = x.float() * rstd
    dw = (dz * unit).sum((0, 1, 2))
    dz = dz * weight.float()
    return (rstd * (dz - unit * (dz * unit).mean(-1, keepdim=True))).to(x.dtype), dw


def _folded(x, c):
    """Query-side tensor [B, H, Lq, d] -> fp32 [B, Hkv, group * Lq, d]: the heads that share keys below each other."""
    return x.float().reshape(c["B"], c["Hkv"], c["group"] * c["Lq"], x.shape[-1])


def _scores(s):
    c = s["case"]
    scores = (_folded(s["q"], c) @ s["k"].float().transpose(2, 3).contiguous()).mul_(s["scale"])
    if s["k_lens"] is not None:
        scores.masked_fill_(torch.arange(c["Lk"], device="cuda") >= s["k_lens"][:, None, None, None], -math.inf)
    return scores


def _plain_cross(s):
    c = s["case"]
    p = _scores(s)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ s["v"].float()) / torch.where(total > 0, total, 1.0)
    shape = (c["B"], c["Hkv"] * c["group"], c["Lq"])
    return out.reshape(*shape, c["d"]).bfloat16(), (top + total.log()).reshape(shape)


def _plain_cross_grad(s):
    c = s["case"]
    lse = s["lse"].reshape(c["B"], c["Hkv"], c["group"] * c["Lq"], 1)
    p = _scores(s).sub_(torch.where(lse == -math.inf, 0.0, lse)).exp_()
    dout = _folded(s["dout"], c)
    dv = p.transpose(2, 3).contiguous() @ dout
    ds = dout @ s["v"].float().transpose(2, 3).contiguous()
    ds = ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    dq = (ds @ s["k"].float()).reshape(c["B"], c["Hkv"] * c["group"], c["Lq"], c["d"])
    dk = ds.transpose(2, 3).contiguous() @ _folded(s["q"], c)
    return dq.bfloat16(), dk.bfloat16(), dv.bfloat16()


def run(s):
    c = s["case"]
    if own:
        return _own(s)
    if c["op"] == "table":
        return _plain_table(s)
    if c["op"] == "rope":
        return _plain_rope(s["q"], s["qw"], s), _plain_rope(s["k"], s["kw"], s)
    if c["op"] == "rope_grad":
        dq, dqw = _plain_rope_grad(s["q"], s["qw"], s["dq_out"], s)
        dk, dkw = _plain_rope_grad(s["k"], s["kw"], s["dk_out"], s)
        return (dq, dk, dqw, dkw) if c["norm"] else (dq, dk)
    return _plain_cross(s) if c["op"] == "cross" else _plain_cross_grad(s)


def _own(s):
    from paper_2509_16518_amd import fgattn as F
    c = s["case"]
    if c["op"] == "table":
        cos = torch.empty((s["rows"], s["pairs"]), dtype=torch.float32, device="cuda")
        sin = torch.empty_like(cos)
        F.fgattn_rope_table(s["axes"], cos, sin, mscale=c["mscale"])
        return cos, sin
    if c["op"] in ("rope", "rope_grad"):
        q, k = s["q"], s["k"]
        layout = F.ROPE_HALF if c["layout"] == "half" else F.ROPE_INTERLEAVED
        flags = F.FLAG_ROPE_NORM if c["norm"] else 0
        a, b = torch.empty_like(q), torch.empty_like(k)
        if c["op"] == "rope":
            p = F.make_rope_params(q, k, a, b, c["rot"], layout, eps=_EPS, flags=flags)
            F.fgattn_rope_forward(q, k, p, a, b, s["cos"], s["sin"], positions=s["positions"], q_weight=s["qw"], k_weight=s["kw"])
            return a, b
        p = F.make_rope_params(q, k, s["dq_out"], s["dk_out"], c["rot"], layout, eps=_EPS, flags=flags)
        if not c["norm"]:
            F.fgattn_rope_backward(q, k, p, s["dq_out"], s["dk_out"], a, b, s["cos"], s["sin"], positions=s["positions"])
            return a, b
        dqw = torch.empty((c["d"],), dtype=torch.float32, device="cuda")
        dkw = torch.empty_like(dqw)
        ws = torch.empty((F.fgattn_rope_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
        F.fgattn_rope_backward(q, k, p, s["dq_out"], s["dk_out"], a, b, s["cos"], s["sin"], positions=s["positions"],
                               q_weight=s["qw"], k_weight=s["kw"], dq_weight=dqw, dk_weight=dkw, workspace=ws)
        return a, b, dqw, dkw
    q, k, v = s["q"], s["k"], s["v"]
    if c["op"] == "cross":
        out = torch.empty_like(q)
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
        p = F.make_cross_params(q, k, v, out, s["scale"])
        ws = torch.empty((F.fgattn_cross_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
        F.fgattn_cross_forward(q, k, v, p, out, lse, ws, k_lens=s["k_lens"])
        return out, lse
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    p = F.make_cross_params(q, k, v, s["out"], s["scale"], s["dout"], dq, dk, dv)
    ws = torch.empty((F.fgattn_cross_backward_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
    F.fgattn_cross_backward(q, k, v, s["out"], s["lse"], s["dout"], p, dq, dk, dv, ws, k_lens=s["k_lens"])
    return dq, dk, dv


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "table":
        return _exact_table(s)
    if c["op"] in ("rope", "rope_grad"):
        found = []
        for x, w, dy in ((s["q"], s["qw"], s.get("dq_out")), (s["k"], s["kw"], s.get("dk_out"))):
            found.append(_exact_rope(x, w, dy, s))
        if c["op"] == "rope":
            return tuple(y for (y,) in found)
        return tuple(dx for dx, _ in found) + (tuple(dw for _, dw in found) if c["norm"] else ())
    return _exact_cross(s)


def _exact_table(s):
    """Every axis by itself as powers of e^(i angle), spread over the grid by broadcasting."""
    sizes = [a[0] for a in s["axes"]]
    turns = []
    for n, (size, pairs, theta, offset, step, factor, original, fast, slow) in enumerate(s["axes"]):
        angles = torch.empty((size, pairs), device="cuda", dtype=torch.float64)
        for j in range(pairs):
            w = math.exp(-j / pairs * math.log(theta))
            turns_trained = original * w / (2 * math.pi)
            share = min(1.0, max(0.0, (turns_trained - slow) / (fast - slow)))
            angles[:, j] = (torch.arange(size, device="cuda", dtype=torch.float64) * step + offset) * (share * w + (1 - share) * w / factor)
        shape = [1] * len(sizes) + [pairs]
        shape[n] = size
        turns.append(torch.polar(torch.full_like(angles, s["case"]["mscale"]), angles).reshape(shape).expand(*sizes, pairs).reshape(s["rows"], pairs))
    z = torch.cat(turns, 1)
    return z.real, z.imag


def _exact_rope(x, w, dy, s):
    """As complex numbers: each pair times e^(i angle); gradients by automatic differentiation of that."""
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    x = x.double().requires_grad_(dy is not None)
    z = x
    if w is not None:
        w = w.double().requires_grad_(dy is not None)
        z = x / (x.pow(2).sum(-1, keepdim=True) / c["d"] + _EPS).sqrt() * w
    if rot:
        turn = torch.complex(s["cos"].double(), s["sin"].double())
        if s["positions"] is not None:
            turn = turn[s["positions"].long()].unsqueeze(1)
        pairs = z[..., :rot].unflatten(-1, (half, 2)) if c["layout"] == "interleaved" else z[..., :rot].unflatten(-1, (2, half)).transpose(-1, -2)
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        turned = turned.flatten(-2) if c["layout"] == "interleaved" else turned.transpose(-1, -2).flatten(-2)
        z = torch.cat((turned, z[..., rot:]), -1)
    if dy is None:
        return (z,)
    grads = torch.autograd.grad(z, (x,) if w is None else (x, w), dy.double())
    return grads if w is not None else (grads[0], None)


def _exact_cross(s):
    """Key head by key head on the keys that count; gradients by automatic differentiation."""
    c = s["case"]
    G, shape = c["group"], s["q"].shape
    grad = c["op"] == "cross_grad"
    result = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in ((s["q"], s["k"], s["v"]) if grad else (s["q"],))]
    lse = torch.full(shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_key_lengths(c)):
        for h in range(c["Hkv"] if n else 0):
            own_heads = slice(h * G, (h + 1) * G)
            q, k, v = (t.double().requires_grad_(grad) for t in (s["q"][b, own_heads], s["k"][b, h, :n], s["v"][b, h, :n]))
            scores = torch.matmul(q.reshape(-1, c["d"]), k.t()) * s["scale"]
            out = torch.softmax(scores, -1) @ v
            if grad:
                dq, dk, dv = torch.autograd.grad(out, (q, k, v), s["dout"][b, own_heads].double().reshape(-1, c["d"]))
                result[0][b, own_heads], result[1][b, h, :n], result[2][b, h, :n] = dq, dk, dv
            else:
                result[0][b, own_heads] = out.reshape(G, c["Lq"], c["d"])
                lse[b, own_heads] = torch.logsumexp(scores, -1).reshape(G, c["Lq"])
    return tuple(result) if grad else (result[0], lse)
