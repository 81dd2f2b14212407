"""Cross attention and its gradients against their 64-bit definitions."""
import math

import pytest
import torch

import plain_ops as P
from paper_2509_16518_amd import fgattn as F

pytestmark = pytest.mark.gpu


def make(gen, storage, B, H, L, d, gain=1.0):
    x = (gain * torch.randn((B, H, L, d), generator=gen, device="cuda")).bfloat16()
    if storage == "blhd":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if storage == "slice":
        wide = torch.full((B, L, H, 2 * d + 24), math.nan, device="cuda").bfloat16()
        wide[..., 8:8 + d] = x.transpose(1, 2)
        return wide[..., 8:8 + d].transpose(1, 2)
    return x


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d off, worst %.3g where %.3g is allowed" % (what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(bound[bad].min()))


def near(got, want, what, limit=2.0 ** -8):
    """Root mean square: roundings of random sign, each at most half a step of bf16, do not add up to half a step on average."""
    norm = float(want.norm())
    if norm:
        assert float((got.double() - want).norm()) <= limit * norm, (what, float((got.double() - want).norm()) / norm)


#        B  Hkv G  Lq   Lk    d   storage scale  q_lens          k_lens
CASES = [
    (1, 1, 1, 1, 1, 64, "bhld", None, None, None),
    (1, 1, 1, 1, 1, 128, "bhld", None, None, None),
    (2, 3, 1, 33, 31, 128, "blhd", None, None, None),
    (2, 3, 1, 32, 32, 64, "slice", None, None, None),
    (1, 2, 1, 130, 33, 128, "bhld", None, None, None),
    (1, 2, 2, 100, 65, 64, "blhd", None, None, None),
    (3, 2, 1, 129, 77, 128, "slice", None, [129, 0, 64], [77, 40, 0]),
    (3, 2, 3, 45, 97, 64, "bhld", 0.3, [1, 45, 32], [1, 97, 64]),
    (4, 1, 5, 7, 300, 128, "blhd", None, [7, 3, 0, 9], [300, 0, -4, 5000]),
    (1, 2, 1, 1, 2000, 128, "bhld", None, None, None),                    # one token, keys split
    (3, 2, 8, 1, 1031, 64, "blhd", None, None, [1031, 128, 1]),
    (2, 4, 5, 1, 8191, 128, "slice", None, None, [8191, 17]),
    (1, 1, 1, 40, 700, 128, "bhld", -0.2, None, None),                    # negative scale
    (1, 2, 1, 50, 90, 64, "bhld", 0.0, None, [90]),                       # scale 0: means
    (2, 12, 1, 1000, 226, 128, "blhd", None, [1000, 777], [226, 199]),    # many rows: 128-row tiles
    (1, 16, 2, 1111, 512, 64, "bhld", None, None, None),
    (1, 40, 1, 900, 1, 128, "bhld", None, None, None),
    (1, 3, 1, 70, 4100, 128, "bhld", None, None, None),
    (2, 12, 1, 1500, 517, 128, "blhd", None, [1500, 1211], [517, 3]),     # many rows, keys beyond what LDS holds: rings
    (3, 6, 2, 1111, 641, 128, "bhld", None, [1111, 1, 600], [384, 641, 0]),
    (1, 9, 4, 1111, 1030, 64, "slice", -0.15, None, None),
    (2, 9, 2, 999, 661, 64, "blhd", None, None, [661, 64]),
    (1, 24, 1, 3001, 320, 128, "bhld", None, None, [289]),                # all of LDS
    (2, 17, 1, 1301, 640, 64, "bhld", None, [1301, 1300], [640, 577]),
    (1, 2, 1, 1, 30011, 128, "bhld", None, None, None),                   # the backward call's ranges of keys, in LDS
    (1, 16, 1, 250, 7000, 128, "blhd", None, [249], [6990]),              # and through rings
    (2, 5, 2, 61, 9001, 64, "bhld", None, None, [9001, 1000]),
    (2, 12, 1, 1100, 128, 128, "bhld", None, None, [128, 1]),             # the last length whose D is summed over the keys
    (2, 3, 1, 400, 129, 64, "blhd", None, None, [129, 2]),
]
IDS = ["-".join(str(x) for x in c[:7]) for c in CASES]


class Problem:
    def __init__(self, case, seed=3, gain=1.0):
        self.B, self.Hkv, self.G, self.Lq, self.Lk, self.d, storage, scale, q_lens, k_lens = case
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.H = self.Hkv * self.G
        self.scale = self.d ** -0.5 if scale is None else scale
        self.q = make(gen, storage, self.B, self.H, self.Lq, self.d, 1.5 * gain)
        self.k, self.v = make(gen, storage, self.B, self.Hkv, self.Lk, self.d), make(gen, "bhld", self.B, self.Hkv, self.Lk, self.d)
        self.dout = make(gen, "blhd", self.B, self.H, self.Lq, self.d, 0.1)
        lens = lambda x: None if x is None else torch.tensor(x, device="cuda", dtype=torch.int32)
        self.q_lens, self.k_lens = lens(q_lens), lens(k_lens)
        for t, n, L in ((self.q, q_lens, self.Lq), (self.dout, q_lens, self.Lq), (self.k, k_lens, self.Lk), (self.v, k_lens, self.Lk)):
            if n is not None:        # what lies past the end may be anything
                for b, m in enumerate(n):
                    t[b, :, max(0, min(m, L)):] = math.nan if b % 2 else math.inf
        self.out = torch.empty_strided(self.q.shape, self.q.stride(), dtype=torch.bfloat16, device="cuda").fill_(99.0)
        self.lse = torch.full((self.B, self.H, self.Lq), 99.0, device="cuda")

    def forward(self):
        p = F.make_cross_params(self.q, self.k, self.v, self.out, self.scale)
        ws = torch.empty(F.fgattn_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
        F.fgattn_cross_forward(self.q, self.k, self.v, p, self.out, self.lse, ws, self.q_lens, self.k_lens)
        return self.out, self.lse

    def backward(self):
        grads = [torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").fill_(99.0) for t in (self.q, self.k, self.v)]
        p = F.make_cross_params(self.q, self.k, self.v, self.out, self.scale, self.dout, *grads)
        ws = torch.empty(F.fgattn_cross_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
        F.fgattn_cross_backward(self.q, self.k, self.v, self.out, self.lse, self.dout, p, *grads, ws, self.q_lens, self.k_lens)
        return grads

    def plain(self, f, *more):
        return f(self.q, self.k, self.v, float(torch.tensor(self.scale, dtype=torch.float32)), *more, q_lens=self.q_lens, k_lens=self.k_lens)


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case):
    x = Problem(case)
    out, lse = x.forward()
    ref, ref_lse, bound, off = x.plain(P.cross_forward)
    assert (out[off] == 99).all() and (lse[off] == 99).all()
    on = ~off
    within(out[on], ref[on], bound[on], "out")
    near(out[on], ref[on], "out")
    empty = ref_lse == -math.inf
    assert (lse[on & empty] == -math.inf).all() and (out[on & empty] == 0).all()
    # fp32 scores: d products and sums; exponentials and their sums to a few steps
    assert ((lse.double() - ref_lse)[on & ~empty].abs() <= 2.0 ** -17 * (1 + ref_lse[on & ~empty].abs())).all()
    first = out.clone(), lse.clone()
    x.forward()
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case):
    x = Problem(case)
    x.forward()
    got = x.backward()
    ref = x.plain(P.cross_backward, x.dout)
    for name, g, (r, bound) in zip(("dq", "dk", "dv"), got, ref):
        within(g, r, bound, name)
        if x.scale and x.Lk > 1:      # (one key: dS = 0 but for roundings)
            near(g, r, name, 2.0 ** -7)
    again = x.backward()
    for a, b in zip(got, again):
        assert torch.equal(a, b)


@pytest.mark.parametrize("gain", [8.0, 40.0])
def test_peaked_scores(gain):
    # scores of hundreds: one key takes nearly all of a row, the exponent base moves, the others vanish
    x = Problem((1, 2, 2, 150, 333, 128, "bhld", None, None, [333]), seed=11, gain=gain)
    out, lse = x.forward()
    s, qq, kk, _, _ = P.cross_parts(x.q, x.k, float(torch.tensor(x.scale, dtype=torch.float32)), None, x.k_lens)
    ref, ref_lse, bound, _ = x.plain(P.cross_forward)
    # an fp32 score of size |s| is off by 2^-24 |q||k| per step of its sum: up to 128 of them
    loose = 128 * 2.0 ** -24 * x.scale * float((qq.abs() @ kk.abs().transpose(2, 3).contiguous()).max())
    within(out, ref, bound + loose * 2 * x.v.double().abs().max(), "out")
    assert ((lse.double() - ref_lse).abs() <= loose + 2.0 ** -20 * ref_lse.abs()).all()
    for g, (r, b) in zip(x.backward(), x.plain(P.cross_backward, x.dout)):
        within(g, r, b + loose * 8 * r.abs().max(), "gradient")


def test_gradient_against_a_difference():
    # the kernels' gradients along a direction against a difference of the 64-bit forward pass along it
    x = Problem((1, 2, 2, 96, 160, 64, "bhld", None, None, [131]), seed=21)
    x.forward()
    grads = x.backward()
    gen = torch.Generator(device="cuda").manual_seed(22)
    value = lambda q, k, v: float((P.cross_forward(q, k, v, x.scale, None, x.k_lens)[0] * x.dout.double()).sum())
    tensors = [t.double() for t in (x.q, x.k, x.v)]
    tensors[1][:, :, 131:] = 0.0
    tensors[2][:, :, 131:] = 0.0
    for n, g in enumerate(grads):
        direction = g.double() / g.double().norm()      # (the steepest: its slope is the gradient's own length)
        moved = lambda h: [t + h * direction if m == n else t for m, t in enumerate(tensors)]
        slope = (value(*moved(1e-4)) - value(*moved(-1e-4))) / 2e-4
        assert math.isclose(slope, float(g.double().norm()), rel_tol=2.0 ** -8), n


def test_graph_with_workspaces_of_its_own():
    x = Problem(CASES[11]), Problem(CASES[6], seed=5)
    for t in x:
        t.forward()
        t.want = [t.out.clone(), t.lse.clone()] + t.backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for t in x:
            t.out.fill_(99.0)
            t.lse.fill_(99.0)
            t.forward()
            t.grads = t.backward()
    for n in range(3):
        for t in x:
            t.v.mul_(2.0)                                   # an exact change: out and dq follow, dv does not
        graph.replay()
        torch.cuda.synchronize()
        for t in x:
            f = 2.0 ** (n + 1)
            off = t.want[0] == 99
            got = torch.where(off, t.want[0], t.out / f)
            assert torch.equal(got, t.want[0]) and torch.equal(t.lse, t.want[1])
            assert torch.equal(t.grads[2], t.want[4])
            assert torch.equal(t.grads[0] / f, t.want[2]) and torch.equal(t.grads[1] / f, t.want[3])


def test_on_a_side_stream():
    x = Problem(CASES[10])
    x.forward()
    want = x.out.clone()
    p = F.make_cross_params(x.q, x.k, x.v, x.out, x.scale)
    ws = torch.empty(F.fgattn_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    x.out.fill_(1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    F.fgattn_cross_forward(x.q, x.k, x.v, p, x.out, x.lse, ws, x.q_lens, x.k_lens, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(x.out, want)


def test_wide_strides():
    # key rows 1 MiB apart: byte offsets inside a slice up to nearly 2^32
    B, H, Lq, Lk, d = 1, 1, 200, 4090, 128
    gen = torch.Generator(device="cuda").manual_seed(6)
    q = make(gen, "bhld", B, H, Lq, d)
    k, v = make(gen, "bhld", B, H, Lk, d), make(gen, "bhld", B, H, Lk, d)
    buf = torch.empty(Lk * 2 ** 19, dtype=torch.bfloat16, device="cuda")
    kw, vw = (buf.as_strided((B, H, Lk, d), (2 ** 19 * Lk, 2 ** 19 * Lk, 2 ** 19, 1), at) for at in (0, 4096))
    kw.copy_(k)
    vw.copy_(v)
    result = []
    for kk, vv in ((k, v), (kw, vw)):
        out, lse = torch.empty_like(q), torch.empty((B, H, Lq), device="cuda")
        p = F.make_cross_params(q, kk, vv, out, d ** -0.5)
        ws = torch.empty(F.fgattn_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        F.fgattn_cross_forward(q, kk, vv, p, out, lse, ws)
        grads = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]
        p = F.make_cross_params(q, kk, vv, out, d ** -0.5, q, *grads)
        ws = torch.empty(F.fgattn_cross_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        F.fgattn_cross_backward(q, kk, vv, out, lse, q, p, *grads, ws)
        result.append([out, lse] + grads)
    for a, b in zip(*result):
        assert torch.equal(a, b)


def test_two_calls_at_once():
    # two problems on two streams, workspaces of their own: each as by itself
    x = Problem(CASES[11], seed=31), Problem(CASES[18], seed=32)
    for t in x:
        t.forward()
        t.want = [t.out.clone(), t.lse.clone()] + t.backward()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [None, None]
    for _ in range(3):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for n, (t, s) in enumerate(zip(x, streams)):
            with torch.cuda.stream(s):
                t.out.fill_(99.0)
                t.forward()
                got[n] = t.backward()
        torch.cuda.synchronize()
        for n, t in enumerate(x):
            for a, b in zip([t.out, t.lse] + got[n], t.want):
                assert torch.equal(a, b)


def test_the_most_keys():
    # nearly 2^24 keys (byte offsets up to 2 GiB), scores 0: the result is the mean of the values, dv the same row everywhere, dk zero
    L, d, rows = 2 ** 24 - 5, 64, 3
    k, v = (torch.empty((1, 1, L, d), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(n)) for n in (1, 2))
    q = torch.zeros((1, 1, rows, d), dtype=torch.bfloat16, device="cuda")
    dout = torch.randn((1, 1, rows, d), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty((1, 1, rows), device="cuda")
    p = F.make_cross_params(q, k, v, out, 0.125)
    F.fgattn_cross_forward(q, k, v, p, out, lse, torch.empty(F.fgattn_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    mean = v.sum(2, dtype=torch.float64) / L
    # 64 ranges of 2^18 keys, 16 keys per matrix instruction: 2^14 additions of fp32 to sums of 2^18 values of size 1 (below 6 * 2^9)
    assert ((out.double() - mean[:, :, None]).abs() <= 2.0 ** -8 * mean.abs()[:, :, None] + 2 ** 14 * 2.0 ** -24 * 6 * 2 ** 9 * 64 / L).all()
    # a logarithm to base 2 near 24, good to one step there (2^-19), times ln 2: 0.7 * 2^-19; that product and its sum with the maximum
    # each rounded near 16.6 (half a step, 2^-20): 1.7 * 2^-19 in all
    assert ((lse.double() - math.log(L)).abs() <= 2.0 ** -18).all()
    grads = [torch.empty_like(t) for t in (q, k, v)]
    p = F.make_cross_params(q, k, v, out, 0.125, dout, *grads)
    F.fgattn_cross_backward(q, k, v, out, lse, dout, p, *grads, torch.empty(F.fgattn_cross_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    assert (grads[1] == 0).all() and torch.isfinite(grads[0]).all()
    dv = dout.double().sum(2) / L
    bound = 2 * 2.0 ** -8 * dout.double().abs().sum(2) / L       # P rounded to bf16, the sum rounded
    for n in range(0, L, 2 ** 21):
        assert ((grads[2][:, :, n:n + 2 ** 21].double() - dv[:, :, None]).abs() <= bound[:, :, None]).all()
