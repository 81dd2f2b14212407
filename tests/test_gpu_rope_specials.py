"""Infinities and NaN in rotary calls: elements that are not turned (behind rot_dims, or of a token without a row in the table) pass
through bit by bit whatever lies beside them, a turned pair stays by itself, and a row's norm stays in its row."""
import math

import pytest
import torch

import plain_ops as P
from paper_2509_16518_amd import fgattn as F

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
EPS = 1e-6
BITS = {BF16: torch.int16, FP16: torch.int16, FP32: torch.int32}

#        L   d   rot  half   dtype  positions
CASES = [
    (7, 64, 48, False, BF16, False),
    (7, 64, 48, True, BF16, False),      # halves of 24: whole chunks
    (9, 96, 36, True, FP16, True),       # halves of 18: partners straddle chunks
    (9, 128, 20, False, FP16, True),     # the end of the turned part inside a chunk
    (5, 256, 128, True, FP32, True),
    (5, 40, 10, False, FP32, True),
    (6, 72, 36, True, FP32, False),      # halves of 18
    (8, 128, 0, False, BF16, False),
    (8, 128, 128, False, BF16, True),    # only the tokens outside the table are not turned
    (8, 128, 128, True, BF16, True),
]
IDS = ["-".join(str(x).replace("torch.", "") for x in c) for c in CASES]
B, HEADS = 2, (3, 2)


def pairs_of(rot, half):
    j = torch.arange(rot // 2)
    return (j, j + rot // 2) if half else (2 * j, 2 * j + 1)


class Setup:
    def __init__(self, case, seed=17):
        self.L, self.d, self.rot, self.half, self.dtype, positions = case
        L, d, rot = self.L, self.d, self.rot
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.cos = self.sin = self.pos = None
        self.layout = F.ROPE_HALF if self.half else F.ROPE_INTERLEAVED
        self.on = torch.zeros((B, L), dtype=torch.bool, device="cuda")       # tokens that are turned
        if rot:
            c, s, _ = P.table([(3 * L, rot // 2, 100.0, 1.0, 1.0, 1.0, 0.0, 32.0, 1.0)])
            self.cos, self.sin = c.float().cuda(), s.float().cuda()
            rows = torch.arange(L, device="cuda").expand(B, L)
            if positions:
                rows = torch.randint(0, 3 * L, (B, L), generator=self.gen, device="cuda")
                rows[0, 1::3] = -1
                rows[1, ::4] = 3 * L
                self.pos = rows.int()
            self.on = (rows >= 0) & (rows < 3 * L)
            self.c, self.s = (t.double()[rows.clamp(0, 3 * L - 1)][:, None] for t in (self.cos, self.sin))
        self.first, self.second = (p.cuda() for p in pairs_of(rot, self.half))

    def values(self, H, special):
        """[B, H, L, d] of which about one element in twelve is infinite or NaN in every second row of every head."""
        x = torch.randn((B, H, self.L, self.d), generator=self.gen, device="cuda").to(self.dtype)
        if special:
            which = torch.rand(x.shape, generator=self.gen, device="cuda")
            which[:, :, ::2] = 1.0
            for n, value in enumerate((math.inf, -math.inf, math.nan, -0.0)):
                x[(which >= 0.02 * n) & (which < 0.02 * (n + 1))] = value
        return x

    def turned(self, z, back=False):
        """z (fp64) turned pair by pair; what is not turned is z itself."""
        y = z.clone()
        if self.rot:
            a, b, s = z[..., self.first], z[..., self.second], -self.s if back else self.s
            on = self.on[:, None, :, None]
            y[..., self.first] = torch.where(on, a * self.c - b * s, a)
            y[..., self.second] = torch.where(on, b * self.c + a * s, b)
        return y

    def still(self, x):
        """The elements of x that are not turned."""
        m = torch.ones_like(x, dtype=torch.bool)
        m[..., :self.rot] = ~self.on[:, None, :, None]
        return m


def close(got, want, limit, what):
    """Equal where the definition gives NaN or an infinity, elsewhere within `limit` of the value (a half step and fp32 work on
    terms of size 8 or less)."""
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), "%s: NaN in %d places, %d expected" % (what, int(got.isnan().sum()), int(want.isnan().sum()))
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]), what
    ok = want.isfinite()
    assert ((got - want)[ok].abs() <= limit * want[ok].abs() + 16 * P.F32 * 16 + 1e-7).all(), what


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_rotation_alone(case):
    t = Setup(case)
    x = [t.values(H, True) for H in HEADS]
    out = [torch.empty_like(v) for v in x]
    p = F.make_rope_params(*x, *out, t.rot, t.layout, EPS, 0)
    F.fgattn_rope_forward(*x, p, *out, t.cos, t.sin, t.pos)
    back = [torch.empty_like(v) for v in x]
    F.fgattn_rope_backward(None, None, F.make_rope_params(*x, *x, t.rot, t.layout, EPS, 0), *x, *back, t.cos, t.sin, t.pos)
    for v, o, g in zip(x, out, back):
        still = t.still(v) & ~v.isnan()
        for y in (o, g):
            assert torch.equal(y[still].view(BITS[t.dtype]), v[still].view(BITS[t.dtype]))
        close(o, t.turned(v.double()), P.HALF[t.dtype], "result")
        close(g, t.turned(v.double(), back=True), P.HALF[t.dtype], "gradient")


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("weighted", [False, True])
def test_with_norm(case, weighted):
    # an infinity makes its row's root mean square infinite: 0 where the row is finite, NaN at the infinity itself and its turned partner
    t = Setup(case)
    x = [t.values(H, True) for H in HEADS]
    w = [(1 + 0.2 * torch.randn(t.d, generator=t.gen, device="cuda")).to(t.dtype) if weighted else None for _ in x]
    if weighted:      # a weight of infinity counts for its own element
        w[0][t.d - 1] = math.inf
    out = [torch.empty_like(v) for v in x]
    p = F.make_rope_params(*x, *out, t.rot, t.layout, EPS, F.FLAG_ROPE_NORM)
    F.fgattn_rope_forward(*x, p, *out, t.cos, t.sin, t.pos, *w)
    for v, o, ww in zip(x, out, w):
        z = v.double() / (v.double().square().mean(-1, keepdim=True) + EPS).sqrt()
        close(o, t.turned(z if ww is None else z * ww.double()), P.HALF[t.dtype], "result")


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_gradients_with_norm(case):
    # incoming gradients with infinities: a row's dx is lost as a whole (its mean is not finite), a weight's gradient only where
    # the turned-back gradient of that very element is
    t = Setup(case)
    x, dy = [t.values(H, False) for H in HEADS], [t.values(H, False) for H in HEADS]
    at = t.d - 2 if t.rot < t.d else 3
    token = int((~t.on[0]).nonzero()[0]) if t.rot == t.d else 2
    for v in dy:
        v[0, 1, token, at] = math.inf
    w = [(1 + 0.2 * torch.randn(t.d, generator=t.gen, device="cuda")).to(t.dtype) for _ in x]
    dx, dw = [torch.empty_like(v) for v in x], [torch.empty(t.d, device="cuda") for _ in x]
    p = F.make_rope_params(*x, *dy, t.rot, t.layout, EPS, F.FLAG_ROPE_NORM)
    ws = torch.empty(F.fgattn_rope_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    F.fgattn_rope_backward(*x, p, *dy, *dx, t.cos, t.sin, t.pos, *w, *dw, workspace=ws)
    for v, g, o, ww, got in zip(x, dy, dx, w, dw):
        dz = t.turned(g.double(), back=True)
        rstd = 1 / (v.double().square().mean(-1, keepdim=True) + EPS).sqrt()
        want = (dz * v.double() * rstd).sum((0, 1, 2))
        assert torch.equal(want.isfinite().nonzero().flatten().cpu(), torch.tensor([e for e in range(t.d) if e != at]))
        size = (dz * v.double() * rstd).abs().sum((0, 1, 2))
        ok = want.isfinite()
        # the sum of at most 90 rows, a term formed with a handful of roundings from two turned parts
        assert torch.equal(got.isfinite(), ok)
        assert ((got.double() - want)[ok].abs() <= (90 + 32) * P.F32 * (size[ok] + 90)).all()
        rows = torch.ones(v.shape[:3], dtype=torch.bool, device="cuda")
        rows[0, 1, token] = False
        u = dz * ww.double()
        unit = v.double() * rstd
        ref = rstd * (u - unit * (u * unit).mean(-1, keepdim=True))
        assert not o[0, 1, token].isfinite().any()
        assert ((o.double() - ref)[rows].abs() <= P.HALF[t.dtype] * ref[rows].abs() + 32 * P.F32 * 64 + 1e-7).all()
