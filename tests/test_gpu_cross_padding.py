"""Padded batches in the gradients of cross attention: zeros behind the lengths whatever the counted rows hold."""
import math

import pytest
import torch

import plain_ops as P
from paper_2509_16518_amd import fgattn as F

pytestmark = pytest.mark.gpu


def lens(x):
    return torch.tensor(x, device="cuda", dtype=torch.int32)


class Call:
    def __init__(self, B, Hkv, G, Lq, Lk, d, q_lens, k_lens, gain=1.5, seed=41):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda H, L, g: (g * torch.randn((B, H, L, d), generator=gen, device="cuda")).bfloat16()
        self.q, self.k, self.v, self.dout = make(Hkv * G, Lq, gain), make(Hkv, Lk, 1.0), make(Hkv, Lk, 1.0), make(Hkv * G, Lq, 0.1)
        self.scale, self.q_lens, self.k_lens = d ** -0.5, lens(q_lens), lens(k_lens)
        self.out = torch.full_like(self.q, 9.0)
        self.lse = torch.full((B, Hkv * G, Lq), 9.0, device="cuda")

    def forward(self):
        p = F.make_cross_params(self.q, self.k, self.v, self.out, self.scale)
        ws = torch.empty(F.fgattn_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
        F.fgattn_cross_forward(self.q, self.k, self.v, p, self.out, self.lse, ws, self.q_lens, self.k_lens)

    def backward(self):
        grads = [torch.full_like(t, 9.0) for t in (self.q, self.k, self.v)]
        p = F.make_cross_params(self.q, self.k, self.v, self.out, self.scale, self.dout, *grads)
        ws = torch.empty(F.fgattn_cross_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
        F.fgattn_cross_backward(self.q, self.k, self.v, self.out, self.lse, self.dout, p, *grads, ws, self.q_lens, self.k_lens)
        return grads


SHAPES = [
    # B Hkv G  Lq  Lk   d    q_lens         k_lens
    (2, 3, 1, 30, 40, 128, [17, 30], [20, 33]),          # one range of rows, resident keys
    (2, 3, 2, 15, 40, 64, [7, 15], [20, 39]),
    (2, 3, 1, 700, 90, 128, [601, 1], [70, 20]),         # rows split over workgroups
    (2, 1, 1, 40, 5000, 128, [33, 2], [4099, 5000]),     # keys split over workgroups
    (2, 65, 1, 30, 350, 128, [21, 30], [333, 17]),       # one range of either, rings
    (2, 65, 1, 30, 700, 64, [21, 30], [661, 17]),
]


@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:6])))
def test_zeros_behind_the_lengths(shape, value):
    # a counted row's incoming gradient and a counted key that are not finite: sums that hold them are lost, the padding stays zero
    x = Call(*shape)
    x.forward()
    q_lens, k_lens = shape[6], shape[7]
    for spoil in ("dout", "k"):
        if spoil == "dout":
            x.dout[0, :, q_lens[0] - 1, 5] = value
        else:
            x.k[0, :, k_lens[0] - 1, 3] = value
        dq, dk, dv = x.backward()
        for b in range(len(q_lens)):
            assert (dq[b, :, q_lens[b]:] == 0).all(), (spoil, b)
            assert (dk[b, :, k_lens[b]:] == 0).all() and (dv[b, :, k_lens[b]:] == 0).all(), (spoil, b)
        # an entry of the batch is lost by itself
        assert dq[1].isfinite().all() and dk[1].isfinite().all() and dv[1].isfinite().all()
