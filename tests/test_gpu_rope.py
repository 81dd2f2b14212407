"""Rotary tables and the norm-with-rotation kernels against their 64-bit definitions, element by element within derived bounds."""
import math

import pytest
import torch

import plain_ops as P
from paper_2509_16518_amd import fgattn as F

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
EPS = 1e-6


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d off, worst %.3g against %.3g" % (what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(bound.expand_as(off)[bad].min()))


AXES = {
    "one": [(1000, 64, 10000.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0)],
    "grid": [(3, 22, 10000.0, 5.0, 1.0, 1.0, 0.0, 32.0, 1.0), (7, 21, 256.0, 0.0, 0.5, 1.0, 0.0, 32.0, 1.0), (13, 21, 10000.0, -2.0, 1.0, 1.0, 0.0, 32.0, 1.0)],
    "single token": [(1, 1, 10000.0, 77.0, 1.0, 1.0, 0.0, 32.0, 1.0)],
    "unit axes": [(1, 3, 100.0, 2.0, 1.0, 1.0, 0.0, 32.0, 1.0), (5, 2, 100.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0), (1, 4, 100.0, 9.0, 1.0, 1.0, 0.0, 32.0, 1.0)],
    "two axes, long rows": [(17, 5, 10000.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0), (333, 6, 500000.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0)],
    "interpolated": [(4097, 32, 10000.0, 0.0, 1.0, 4.0, 0.0, 32.0, 1.0)],
    "scaled by wavelength": [(118800, 64, 1e6, 100000.0, 1.0, 8.0, 16384.0, 32.0, 1.0)],
    "steps back": [(100, 128, 10000.0, 50.0, -0.25, 1.0, 0.0, 32.0, 1.0)],
}


@pytest.mark.parametrize("name", sorted(AXES))
@pytest.mark.parametrize("mscale", [1.0, 1.2079])
def test_table(name, mscale):
    axes = AXES[name]
    rows, pairs = math.prod(a[0] for a in axes), sum(a[1] for a in axes)
    cos, sin = (torch.full((rows + 1, pairs), 7.0, device="cuda") for _ in "cs")
    F.fgattn_rope_table(axes, cos[:rows], sin[:rows], mscale=mscale)
    c, s, angle = P.table(axes, mscale)
    # one rounding to fp32; angles and 16 turns in 64 bits (each to a few steps of the angle, both sides)
    slack = mscale * (angle.abs() * 2.0 ** -48 + 2.0 ** -44)
    within(cos[:rows].cpu(), c, P.F32 * c.abs() + slack, name)
    within(sin[:rows].cpu(), s, P.F32 * s.abs() + slack, name)
    assert (cos[rows] == 7).all() and (sin[rows] == 7).all()


def test_table_defaults():
    cos, sin = torch.empty((9, 4), device="cuda"), torch.empty((9, 4), device="cuda")
    F.fgattn_rope_table([(9, 4, 100.0)], cos, sin)
    c, s, _ = P.table([(9, 4, 100.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0)])
    within(cos.cpu(), c, torch.tensor(2.0 ** -24), "cos")
    within(sin.cpu(), s, torch.tensor(2.0 ** -24), "sin")


def make(gen, storage, B, H, L, d, dtype, gain=1.0):
    """[B, H, L, d] tensors that lie in memory in different ways."""
    x = (gain * torch.randn((B, H, L, d), generator=gen, device="cuda")).to(dtype)
    if storage == "blhd":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if storage == "slice":   # of a wider projection, rows further apart than a row is long
        wide = torch.full((B, L, H, 3 * d + 8), 1e4, device="cuda").to(dtype)
        wide[..., d:2 * d] = x.transpose(1, 2)
        return wide[..., d:2 * d].transpose(1, 2)
    return x


#        B  Hq Hk  L    d   rot  half  dtype  norm  positions weight       storage
CASES = [
    (1, 1, 1, 1, 128, 128, False, BF16, True, None, "same", "bhld"),
    (2, 3, 1, 5, 64, 64, False, BF16, True, None, "same", "blhd"),
    (2, 3, 2, 37, 128, 128, True, BF16, True, "any", "fp32", "slice"),
    (1, 12, 12, 300, 128, 96, False, BF16, True, None, "same", "bhld"),
    (1, 5, 5, 77, 128, 48, True, FP16, True, "outside", "same", "blhd"),
    (3, 2, 2, 19, 96, 72, True, FP16, True, None, None, "bhld"),           # halves of 36: partners straddle chunks
    (1, 4, 2, 65, 64, 20, True, BF16, False, "any", None, "slice"),        # halves of 10
    (1, 4, 4, 50, 256, 256, True, BF16, True, None, "same", "bhld"),
    (1, 2, 2, 33, 256, 250, False, FP32, True, None, "same", "blhd"),
    (2, 2, 2, 21, 128, 100, True, FP32, True, "any", "same", "bhld"),      # halves of 50
    (2, 3, 3, 40, 64, 64, True, FP32, False, None, None, "slice"),
    (1, 3, 3, 40, 32, 16, False, FP32, True, None, "same", "bhld"),
    (2, 1, 1, 9, 8, 8, False, BF16, True, None, "same", "blhd"),
    (2, 2, 2, 9, 8, 2, True, FP16, True, "any", "same", "bhld"),
    (1, 6, 2, 31, 40, 40, False, FP16, False, None, None, "bhld"),
    (2, 7, 3, 23, 72, 0, False, BF16, True, None, "same", "blhd"),         # the norm alone
    (1, 2, 0, 90, 128, 128, False, BF16, True, None, "same", "bhld"),      # queries alone
    (1, 40, 8, 1, 128, 128, True, BF16, True, "any", "same", "blhd"),      # one token
    (4, 2, 2, 700, 128, 64, False, FP16, True, "any", "fp32", "blhd"),
]


def problem(case, seed=5):
    B, Hq, Hk, L, d, rot, half, dtype, norm, positions, weight, storage = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = [make(gen, storage, B, Hq, L, d, dtype, 2.0), make(gen, storage, B, Hk, L, d, dtype, 0.1) if Hk else None]
    dy = [make(gen, "blhd", B, Hq, L, d, dtype, 0.5), make(gen, "bhld", B, Hk, L, d, dtype, 3.0) if Hk else None]
    w = [None, None]
    if norm and weight:
        w = [(1 + 0.5 * torch.randn(d, generator=gen, device="cuda")).to(FP32 if weight == "fp32" else dtype) for _ in "qk"]
        if not Hk:
            w[1] = None
    rows = 3 * L + 4 if positions else L
    cos = sin = pos = None
    if rot:
        c, s, _ = P.table([(rows, rot // 2, 10000.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0)], 1.1)
        cos, sin = c.float().cuda(), s.float().cuda()
        if positions:
            pos = torch.randint(0, rows, (B, L), generator=gen, device="cuda", dtype=torch.int32)
            if positions == "outside":
                pos[0, ::3] = -1
                pos[0, 1::7] = rows
    flags = (F.FLAG_ROPE_NORM if norm else 0) | (F.FLAG_ROPE_WEIGHT_FP32 if weight == "fp32" else 0)
    R = P.turn_matrix(cos, sin, pos, d, rot, half, L).cuda()
    return x, dy, w, cos, sin, pos, flags, R


def out_like(x, fill):
    return None if x is None else torch.full_like(x, fill)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_forward(case):
    d, rot, half, norm = case[4], case[5], case[6], case[8]
    x, _, w, cos, sin, pos, flags, R = problem(case)
    layout = F.ROPE_HALF if half else F.ROPE_INTERLEAVED
    out = [out_like(t, 99.0) for t in x]
    p = F.make_rope_params(*x, *out, rot, layout, EPS, flags)
    F.fgattn_rope_forward(*x, p, *out, cos, sin, pos, *w)
    eps = float(torch.tensor(EPS, dtype=FP32))
    for t, o, ww in zip(x, out, w):
        if t is not None:
            y, bound = P.rope_forward(t, ww, R, eps, norm)
            within(o, y, bound, "result")
    again = [None if t is None else t.clone(memory_format=torch.preserve_format) for t in x]   # in place
    for a, t in zip(again, x):
        if t is not None:
            a.copy_(t)
    p = F.make_rope_params(*again, *again, rot, layout, EPS, flags)
    F.fgattn_rope_forward(*again, p, *again, cos, sin, pos, *w)
    for a, o in zip(again, out):
        assert a is None or torch.equal(a, o)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_backward(case):
    d, rot, half, norm = case[4], case[5], case[6], case[8]
    x, dy, w, cos, sin, pos, flags, R = problem(case)
    layout = F.ROPE_HALF if half else F.ROPE_INTERLEAVED
    dx = [None if t is None else torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").fill_(99.0) for t in x]
    p = F.make_rope_params(*x, *dy, rot, layout, EPS, flags)
    dw = [torch.full((d,), 99.0, device="cuda") if norm and t is not None else None for t in x]
    ws = torch.empty(F.fgattn_rope_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
    F.fgattn_rope_backward(*x, p, *dy, *dx, cos, sin, pos, *w, *dw, workspace=ws)
    eps = float(torch.tensor(EPS, dtype=FP32))
    first = [None if t is None else t.clone() for t in dx + dw]
    for t, g, o, ww, gw in zip(x, dy, dx, w, dw):
        if t is None:
            continue
        ref, bound, ref_w, bound_w = P.rope_backward(t, ww, R, eps, norm, g)
        within(o, ref, bound, "gradient")
        if norm:
            within(gw, ref_w, bound_w, "weight gradient")
    # no weight gradients wanted: no workspace; the same bits a second time; without the norm the inputs are not read
    F.fgattn_rope_backward(*x, p, *dy, *dx, cos, sin, pos, *w)
    for a, b in zip(dx, first):
        assert a is None or torch.equal(a, b)
    F.fgattn_rope_backward(*x, p, *dy, *dx, cos, sin, pos, *w, *dw, workspace=ws)
    for a, b in zip(dx + dw, first):
        assert a is None or torch.equal(a, b)
    if not norm:
        F.fgattn_rope_backward(None, None, p, *dy, *dx, cos, sin, pos)
        for a, b in zip(dx, first):
            assert a is None or torch.equal(a, b)


def test_broadcast_input_and_rows_between():
    # q read with stride 0 over the batch; the rows of a wider buffer that are not the result's stay as they were
    gen = torch.Generator(device="cuda").manual_seed(8)
    base = torch.randn((1, 3, 17, 64), generator=gen, device="cuda").bfloat16()
    q = base.expand(4, 3, 17, 64)
    wide = torch.full((4, 3, 40, 64), 5.0, device="cuda").bfloat16()
    out = wide[:, :, 11:28]
    cos, sin = torch.empty((17, 32), device="cuda"), torch.empty((17, 32), device="cuda")
    F.fgattn_rope_table([(17, 32, 10000.0)], cos, sin)
    p = F.make_rope_params(q, None, out, None, 64)
    F.fgattn_rope_forward(q, None, p, out, None, cos, sin)
    y, bound = P.rope_forward(q, None, P.turn_matrix(cos, sin, None, 64, 64, False, 17), EPS, True)
    within(out, y, bound, "result")
    assert (wide[:, :, :11] == 5).all() and (wide[:, :, 28:] == 5).all()


def test_many_tokens_and_offsets_past_32_bits():
    # two tokens 6 GiB apart in a buffer that only they touch
    far = 3 * 2 ** 30 // 8 * 8
    buf = torch.empty(far + 4096, dtype=BF16, device="cuda")
    x = buf.as_strided((2, 2, 3, 64), (far, 512, 128, 1))
    gen = torch.Generator(device="cuda").manual_seed(9)
    x.copy_(torch.randn((2, 2, 3, 64), generator=gen, device="cuda"))
    ref = x.clone()
    c, s, _ = P.table([(3, 32, 100.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0)])
    cos, sin = c.float().cuda(), s.float().cuda()
    p = F.make_rope_params(x, None, x, None, 64)
    F.fgattn_rope_forward(x, None, p, x, None, cos, sin)
    y, bound = P.rope_forward(ref, None, P.turn_matrix(cos, sin, None, 64, 64, False, 3), EPS, True)
    within(x, y, bound, "result")


def test_graph_and_streams():
    case = CASES[3]
    x, dy, w, cos, sin, pos, flags, R = problem(case)
    out, dx = [torch.empty_like(t) for t in x], [torch.empty_like(t) for t in x]
    dw = [torch.empty(128, device="cuda") for _ in x]
    p, pb = F.make_rope_params(*x, *out, case[5], 0, EPS, flags), F.make_rope_params(*x, *dy, case[5], 0, EPS, flags)
    ws = torch.empty(F.fgattn_rope_workspace_bytes(pb), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        F.fgattn_rope_forward(*x, p, *out, cos, sin, pos, *w, stream=stream)
        F.fgattn_rope_backward(*x, pb, *dy, *dx, cos, sin, pos, *w, *dw, workspace=ws, stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    want = [t.clone() for t in out + dx + dw]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(3):
        for t in x:
            t.mul_(-1.0)      # results turn their signs; the weights' gradients do not (x and dy enter once each)
        for t in out + dx + dw:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        sign = -1.0 if n % 2 == 0 else 1.0
        for t, v in zip(out, want[:2]):
            assert torch.equal(t, sign * v)
        for t, v in zip(dx, want[2:4]):
            assert torch.equal(t, v)
        for t, v in zip(dw, want[4:]):
            assert torch.equal(t, sign * v)
