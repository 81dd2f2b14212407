"""Plain definitions, in 64 bits, of the operators around the sparse attention (rotary tables, norm with rotation, cross attention) and
of their gradients, with bounds on what a kernel may be off by.  Written from the formulas in include/fgattn.h."""
import math

import torch

# half a step of each type, relative to the value
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# half the smallest positive value (what a result near zero may lose)
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}
F32 = 2.0 ** -24


def table(axes, mscale=1.0):
    """axes: (size, pairs, theta, offset, step, factor, original, beta_fast, beta_slow)"""
    sizes = [a[0] for a in axes]
    columns = []
    for n, (size, pairs, theta, offset, step, factor, original, fast, slow) in enumerate(axes):
        w = torch.tensor([theta ** (-j / pairs) for j in range(pairs)], dtype=torch.float64)
        keep = ((original * w / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1) if original > 0 else torch.zeros_like(w)
        angle = (offset + step * torch.arange(size, dtype=torch.float64))[:, None] * (w * (keep + (1 - keep) / factor))
        view = [1] * len(sizes) + [pairs]
        view[n] = size
        columns.append(angle.view(view).expand(*sizes, pairs).reshape(-1, pairs))
    angle = torch.cat(columns, 1)
    return mscale * angle.cos(), mscale * angle.sin(), angle


def turn_matrix(cos, sin, positions, d, rot, half_layout, L):
    """[B or 1, L, d, d] matrices R with y = R z, from the fp32 table."""
    if positions is None:
        positions = torch.arange(L, device=cos.device)[None] if rot else torch.zeros((1, L), dtype=torch.int64)
    rows = positions.long()
    R = torch.zeros((*rows.shape, d, d), dtype=torch.float64, device=rows.device)
    R += torch.eye(d, dtype=torch.float64, device=rows.device)
    if rot:
        ok = (rows >= 0) & (rows < cos.shape[0])
        c, s = cos.double()[rows.clamp(0, cos.shape[0] - 1)], sin.double()[rows.clamp(0, cos.shape[0] - 1)]
        c, s = torch.where(ok[..., None], c, 1.0), torch.where(ok[..., None], s, 0.0)
        for j in range(rot // 2):
            a, b = (j, j + rot // 2) if half_layout else (2 * j, 2 * j + 1)
            R[..., a, a], R[..., a, b] = c[..., j], -s[..., j]
            R[..., b, b], R[..., b, a] = c[..., j], s[..., j]
    return R


def rope_forward(x, weight, R, eps, norm):
    """x [B, H, L, d] -> (y, bound) in 64 bits; bound: largest error of a kernel that works in fp32 and rounds once to x's type."""
    z = x.double()
    if norm:
        z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt()
        if weight is not None:
            z = z * weight.double()
    y = (R[:, None] @ z[..., None])[..., 0]
    # the mean of squares: a chain of at most 13 roundings, halved by the root; root, weight, product with cosine and sum: 7
    size = (R[:, None].abs() @ z.abs()[..., None])[..., 0]
    return y, HALF[x.dtype] * y.abs() + 16 * F32 * size + TINY[x.dtype]


def rope_backward(x, weight, R, eps, norm, dy):
    """-> (dx, bound, dw, bound of dw)"""
    back = R.transpose(-1, -2)[:, None]
    dz = (back @ dy.double()[..., None])[..., 0]
    size = (back.abs() @ dy.double().abs()[..., None])[..., 0]
    if not norm:
        return dz, HALF[dy.dtype] * dz.abs() + 16 * F32 * size + TINY[dy.dtype], None, None
    rstd = 1 / (x.double().square().mean(-1, keepdim=True) + eps).sqrt()
    unit = x.double() * rstd
    w = torch.ones_like(x[0, 0, 0]).double() if weight is None else weight.double()
    dw = (dz * unit).sum((0, 1, 2))
    u, u_size = dz * w, size * w.abs()
    dx = rstd * (u - unit * (u * unit).mean(-1, keepdim=True))
    inner = u_size + unit.abs() * (u_size * unit.abs()).mean(-1, keepdim=True)
    rows = x[..., 0].numel()
    # a weight gradient's longest chain of additions: a quarter of the rows in one lane, then the workgroup and the workgroups
    return dx, HALF[dy.dtype] * dx.abs() + 32 * F32 * rstd * inner + TINY[dy.dtype], dw, (rows / 4 + 120) * F32 * (size * unit.abs()).sum((0, 1, 2)) + 1e-30


def cross_parts(q, k, scale, q_lens, k_lens):
    """Scores [B, H, Lq, Lk] in 64 bits, -inf where a key does not count, and the keys spread over their query heads."""
    G = q.shape[1] // k.shape[1]
    B, _, Lk, _ = k.shape
    dead = torch.zeros((B, Lk), dtype=torch.bool, device=k.device)
    if k_lens is not None:
        dead = torch.arange(Lk, device=k.device)[None] >= k_lens[:, None]
    kk = torch.where(dead[:, None, :, None], 0.0, k.double()).repeat_interleave(G, 1)
    off = torch.zeros(q.shape[:3], dtype=torch.bool, device=q.device)
    if q_lens is not None:
        off |= (torch.arange(q.shape[2], device=q.device)[None] >= q_lens[:, None])[:, None]
    qq = torch.where(off[..., None], 0.0, q.double())
    s = (qq @ kk.transpose(2, 3).contiguous()) * scale
    s = s.masked_fill(dead[:, None, None], -math.inf)
    return s, qq, kk, dead, off


def values(v, dead, G):
    return torch.where(dead[:, None, :, None], 0.0, v.double()).repeat_interleave(G, 1)


def cross_forward(q, k, v, scale, q_lens=None, k_lens=None):
    """-> (out, lse, bound of out, rows that do not count)"""
    s, _, _, dead, off = cross_parts(q, k, scale, q_lens, k_lens)
    vv = values(v, dead, q.shape[1] // k.shape[1])
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    out = p @ vv
    # a probability is rounded to bf16 once, the result once; fp32 scores, exponentials and sums: 2^-12 between them
    bound = (2.0 ** -8 + 2.0 ** -12) * (p @ vv.abs()) + 2.0 ** -8 * out.abs() + 1e-30
    return out, lse, bound, off


def cross_backward(q, k, v, scale, dout, q_lens=None, k_lens=None):
    """-> three (gradient, bound)"""
    G = q.shape[1] // k.shape[1]
    B, Hkv, Lk, d = k.shape
    s, qq, kk, dead, off = cross_parts(q, k, scale, q_lens, k_lens)
    vv = values(v, dead, G)
    do = torch.where(off[..., None], 0.0, dout.double())
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    p = torch.where(off[..., None], 0.0, p)
    out = p @ vv
    dp = do @ vv.transpose(2, 3).contiguous()
    delta = (do * out).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    # per score: dS rounded to bf16; D from the bf16 result (each product of the sum off by half a step of out); fp32 work
    e = 2.0 ** -8
    err = (e + 2.0 ** -11) * ds.abs() + p * (e * (do * out).abs().sum(-1, keepdim=True) + 2.0 ** -11 * (do.abs() @ vv.abs().transpose(2, 3).contiguous()))
    t = lambda m: m.transpose(2, 3).contiguous()
    heads = lambda m: m.view(B, Hkv, G, Lk, d).sum(2)
    dq, dq_err = scale * (ds @ kk), abs(scale) * (err @ kk.abs())
    dk, dk_err = scale * heads(t(ds) @ qq), abs(scale) * heads(t(err) @ qq.abs())
    dv, dv_err = heads(t(p) @ do), (e + 2.0 ** -11) * heads(t(p) @ do.abs())
    # (2^-126: what bf16 loses near zero)
    return tuple((g, b + e * g.abs() + 2.0 ** -126) for g, b in ((dq, dq_err), (dk, dk_err), (dv, dv_err)))
