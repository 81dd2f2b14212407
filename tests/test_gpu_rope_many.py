"""Rotary calls with so many tokens that a workgroup goes through several tiles of them, and a share of the heads that takes its loop
several steps and reaches from the queries' heads into the keys'."""
import pytest
import torch

import plain_ops as P
from paper_2509_16518_amd import fgattn as F

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
EPS = 1e-6

#        B  Hq Hk  L     d   rot  half   dtype  rows of a workgroup
CASES = [
    (2, 7, 2, 9001, 128, 128, False, BF16, 16),      # 1126 tiles of tokens (the last one short), nine heads in shares of five
    (2, 5, 4, 17003, 64, 48, True, FP16, 32),        # halves of 24
    (1, 2, 7, 17005, 96, 36, True, BF16, 16),        # halves of 18
    (3, 6, 3, 1501, 256, 250, False, FP32, 4),
]
IDS = ["-".join(str(x).replace("torch.", "") for x in c) for c in CASES]


class Setup:
    def __init__(self, case):
        B, Hq, Hk, L, d, rot, self.half, dtype, rows = case
        gen = torch.Generator(device="cuda").manual_seed(61)
        make = lambda H, g: (g * torch.randn((B, L, H, d), generator=gen, device="cuda")).to(dtype).transpose(1, 2)
        self.x, self.dy = [make(Hq, 2.0), make(Hk, 0.5)], [make(Hq, 0.5), make(Hk, 2.0)]
        self.w = [(1 + 0.3 * torch.randn(d, generator=gen, device="cuda")).to(dtype) for _ in "qk"]
        c, s, _ = P.table([(2 * L, rot // 2, 10000.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0)])
        self.cos, self.sin = c.float().cuda(), s.float().cuda()
        self.pos = torch.randint(0, 2 * L, (B, L), generator=gen, device="cuda", dtype=torch.int32)
        self.layout = F.ROPE_HALF if self.half else F.ROPE_INTERLEAVED
        self.rot, self.d = rot, d
        j = torch.arange(rot // 2, device="cuda")
        self.at = (j, j + rot // 2) if self.half else (2 * j, 2 * j + 1)

    def turned(self, z, back=False):
        """-> (z turned, the sum of the sizes of each element's terms)"""
        a, b = z[..., self.at[0]], z[..., self.at[1]]
        c, s = self.cos.double()[self.pos.long()][:, None], self.sin.double()[self.pos.long()][:, None]
        s = -s if back else s
        y, size = z.clone(), z.abs()
        y[..., self.at[0]], y[..., self.at[1]] = a * c - b * s, b * c + a * s
        size[..., self.at[0]], size[..., self.at[1]] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
        return y, size


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert int(bad.sum()) == 0, "%s: %d of %d off, worst %.3g of what is allowed" % (what, int(bad.sum()), bad.numel(), float((off / bound)[bad].max()))


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case):
    t, dtype = Setup(case), case[7]
    out = [torch.empty_like(v) for v in t.x]
    p = F.make_rope_params(*t.x, *out, t.rot, t.layout, EPS)
    F.fgattn_rope_forward(*t.x, p, *out, t.cos, t.sin, t.pos, *t.w)
    for v, o, w in zip(t.x, out, t.w):
        z = v.double() / (v.double().square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()
        y, size = t.turned(z)
        within(o, y, P.HALF[dtype] * y.abs() + 16 * P.F32 * size + P.TINY[dtype], "result")
    again = [v.clone() for v in t.x]
    F.fgattn_rope_forward(*again, F.make_rope_params(*again, *again, t.rot, t.layout, EPS), *again, t.cos, t.sin, t.pos, *t.w)
    for a, o in zip(again, out):
        assert torch.equal(a, o)


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case):
    t, (B, Hq, Hk, L, d, _, _, dtype, rows) = Setup(case), case
    dx, dw = [torch.empty_like(v) for v in t.x], [torch.full((d,), 9.0, device="cuda") for _ in "qk"]
    p = F.make_rope_params(*t.x, *t.dy, t.rot, t.layout, EPS)
    tiles, heads = -(-B * L // rows), 5
    # 1024 workgroups for each of two shares of the heads: tiles and heads are gone through in steps
    assert tiles > 1024 and F.fgattn_rope_workspace_bytes(p) == 1024 * 2 * 2 * d * 4
    ws = torch.empty(F.fgattn_rope_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
    run = lambda: F.fgattn_rope_backward(*t.x, p, *t.dy, *dx, t.cos, t.sin, t.pos, *t.w, *dw, workspace=ws)
    run()
    # a weight gradient's longest chain of additions: the tiles and heads of a lane, the lanes of a workgroup, a 64th of the 2048
    # workgroups, 64 slices pairwise; each term is formed with 16 roundings
    chain = -(-tiles // 1024) * heads + rows + 2048 // 64 + 6 + 16
    for v, g, o, w, got in zip(t.x, t.dy, dx, t.w, dw):
        dz, size = t.turned(g.double(), back=True)
        rstd = 1 / (v.double().square().mean(-1, keepdim=True) + EPS).sqrt()
        unit = v.double() * rstd
        within(got, (dz * unit).sum((0, 1, 2)), chain * P.F32 * (size * unit.abs()).sum((0, 1, 2)), "weight gradient")
        u, u_size = dz * w.double(), size * w.double().abs()
        ref = rstd * (u - unit * (u * unit).mean(-1, keepdim=True))
        inner = u_size + unit.abs() * (u_size * unit.abs()).mean(-1, keepdim=True)
        within(o, ref, P.HALF[dtype] * ref.abs() + 32 * P.F32 * rstd * inner + P.TINY[dtype], "gradient")
    first = [v.clone() for v in dx + dw]
    run()
    for a, b in zip(dx + dw, first):
        assert torch.equal(a, b)
