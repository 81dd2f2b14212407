"""The operators of a layer one after the other, as a video transformer's block runs them: angles of the token grid, norm and rotation of
queries and keys, the mask from their block means, the sparse forward pass, then cross attention to a padded text; and the
gradients of the parts that have them."""
import numpy as np
import pytest
import torch

import plain_ops as P
from gpu_util import OUT_MAX_ABS, OUT_MEAN_ABS, out_to_f64
from paper_2509_16518_amd import fgattn as F

pytestmark = pytest.mark.gpu


def layer(B, H, grid, d, text, x):
    """x: q, k, v (tokens first in memory), norm weights, text q / k / v and lengths; returns everything on the way."""
    T, Hg, Wg = grid
    L = T * Hg * Wg
    pairs = d // 2
    a = pairs - 2 * (pairs // 3)
    cos, sin = torch.empty((L, pairs), device="cuda"), torch.empty((L, pairs), device="cuda")
    F.fgattn_rope_table([(T, a, 10000.0), (Hg, pairs // 3, 10000.0), (Wg, pairs // 3, 10000.0)], cos, sin)
    qr, kr = torch.empty_like(x["q"]), torch.empty_like(x["k"])
    rp = F.make_rope_params(x["q"], x["k"], qr, kr, d)
    F.fgattn_rope_forward(x["q"], x["k"], rp, qr, kr, cos, sin, q_weight=x["qw"], k_weight=x["kw"])
    out, lse = torch.empty_like(x["q"]), torch.empty((B, H, L), device="cuda")
    M, N = 64, 32
    p = F.make_params(qr, kr, x["v"], out, M, N, d ** -0.5)
    mws = torch.empty(F.fgattn_mask_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    items = B * H * -(-L // M)
    indptr = torch.empty(items + 1, dtype=torch.int64, device="cuda")
    F.fgattn_mask_select(qr, kr, p, 0.9, indptr, mws)
    indices = torch.full((items * -(-L // N),), -1, dtype=torch.int32, device="cuda")
    F.fgattn_mask_emit(p, indptr, indices, mws)
    ws = torch.empty(F.fgattn_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    F.fgattn_forward(qr, kr, x["v"], indptr, indices, p, out, lse, ws)
    # cross attention: queries normed alone (no rotation), keys of the text normed in a call of their own
    cq, ck = torch.empty_like(x["cq"]), torch.empty_like(x["ck"])
    F.fgattn_rope_forward(x["cq"], None, F.make_rope_params(x["cq"], None, cq, None, 0), cq, None, q_weight=x["qw"])
    F.fgattn_rope_forward(x["ck"], None, F.make_rope_params(x["ck"], None, ck, None, 0), ck, None, q_weight=x["kw"])
    cout, clse = torch.empty_like(cq), torch.empty((B, H, L), device="cuda")
    cp = F.make_cross_params(cq, ck, x["cv"], cout, d ** -0.5)
    cws = torch.empty(F.fgattn_cross_workspace_bytes(cp), dtype=torch.uint8, device="cuda")
    F.fgattn_cross_forward(cq, ck, x["cv"], cp, cout, clse, cws, k_lens=x["lens"])
    return dict(cos=cos, sin=sin, qr=qr, kr=kr, indptr=indptr, indices=indices, out=out, lse=lse, cq=cq, ck=ck, cout=cout, clse=clse)


@pytest.mark.parametrize("d,H", [(128, 3), (64, 2)])
def test_block(d, H):
    B, grid, text = 2, (3, 9, 14), 61
    L = grid[0] * grid[1] * grid[2]
    gen = torch.Generator(device="cuda").manual_seed(d)
    tokens = lambda n, gain: (gain * torch.randn((B, n, H, d), generator=gen, device="cuda")).bfloat16().transpose(1, 2)
    weight = lambda: (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).bfloat16()
    x = dict(q=tokens(L, 3.0), k=tokens(L, 0.5), v=tokens(L, 1.0), qw=weight(), kw=weight(), cq=tokens(L, 1.0), ck=tokens(text, 2.0),
             cv=tokens(text, 1.0), lens=torch.tensor([text, 23], dtype=torch.int32, device="cuda"))
    r = layer(B, H, grid, d, text, x)
    # each step against its definition on the step's own inputs
    R = P.turn_matrix(r["cos"], r["sin"], None, d, d, False, L)
    for name, w in (("q", "qw"), ("k", "kw")):
        y, bound = P.rope_forward(x[name], x[w], R, 1e-6, True)
        assert ((r[name + "r"].double() - y).abs() <= bound).all()
    indptr, ids = r["indptr"].cpu().numpy(), r["indices"].cpu().numpy()
    assert (np.diff(indptr) > 0).all()
    M, N, QB = 64, 32, -(-L // 64)
    keep = torch.zeros((B * H, L, L), dtype=torch.bool)
    for w in range(B * H * QB):
        s, i = divmod(w, QB)
        for g in ids[indptr[w]:indptr[w + 1]]:
            keep[s, i * M:(i + 1) * M, g * N:(g + 1) * N] = True
    scores = (r["qr"].double().cpu() @ r["kr"].double().cpu().transpose(2, 3)) * d ** -0.5
    scores = scores.masked_fill(~keep.view(B, H, L, L), float("-inf"))
    off = np.abs(out_to_f64(r["out"]) - (torch.softmax(scores, -1) @ x["v"].double().cpu()).numpy())
    assert off.max() <= OUT_MAX_ABS and off.mean() <= OUT_MEAN_ABS
    for name, w in (("cq", "qw"), ("ck", "kw")):
        y, bound = P.rope_forward(x[name], x[w], torch.eye(d, dtype=torch.float64, device="cuda").expand(1, x[name].shape[2], d, d), 1e-6, True)
        assert ((r[name].double() - y).abs() <= bound).all()
    ref, _, bound, _ = P.cross_forward(r["cq"], r["ck"], x["cv"], d ** -0.5, None, x["lens"])
    assert ((r["cout"].double() - ref).abs() <= bound).all()

    # the way back from the cross attention's result to its un-normed queries, against the definitions chained in 64 bits
    dout = (0.1 * torch.randn((B, H, L, d), generator=gen, device="cuda")).bfloat16()
    dcq, dck, dcv = torch.empty_like(r["cq"]), torch.empty_like(r["ck"]), torch.empty_like(x["cv"])
    cp = F.make_cross_params(r["cq"], r["ck"], x["cv"], r["cout"], d ** -0.5, dout, dcq, dck, dcv)
    ws = torch.empty(F.fgattn_cross_backward_workspace_bytes(cp), dtype=torch.uint8, device="cuda")
    F.fgattn_cross_backward(r["cq"], r["ck"], x["cv"], r["cout"], r["clse"], dout, cp, dcq, dck, dcv, ws, k_lens=x["lens"])
    dx, dw = torch.empty_like(x["cq"]), torch.empty(d, device="cuda")
    rp = F.make_rope_params(x["cq"], None, dcq, None, 0)
    rws = torch.empty(F.fgattn_rope_workspace_bytes(rp), dtype=torch.uint8, device="cuda")
    F.fgattn_rope_backward(x["cq"], None, rp, dcq, None, dx, None, q_weight=x["qw"], dq_weight=dw, workspace=rws)
    leaf, wl = x["cq"].double().requires_grad_(), x["qw"].double().requires_grad_()
    z = leaf / (leaf.square().mean(-1, keepdim=True) + 1e-6).sqrt() * wl
    s = (z @ r["ck"].double().transpose(2, 3).contiguous()) * d ** -0.5
    s = s.masked_fill(torch.arange(text, device="cuda") >= x["lens"][:, None, None, None], float("-inf"))
    gx, gw = torch.autograd.grad(torch.softmax(s, -1) @ torch.where(torch.arange(text, device="cuda")[:, None] < x["lens"][:, None, None, None],
                                                                   x["cv"].double(), 0.0), (leaf, wl), dout.double())
    # four roundings to bf16 on the way (z, out, dS, dcq, dx), each at most 2^-8 and of random sign
    for got, want in ((dx, gx), (dw, gw)):
        assert float((got.double() - want).norm()) <= 4 * 2.0 ** -8 * float(want.norm())
    torch.cuda.synchronize()
