"""Gradients of cross attention with few keys, in batches that are padded further: their accuracy goes by the keys that an entry has and not
by the length that its batch is padded to."""
import math

import pytest
import torch

import plain_ops as P
from test_gpu_cross_padding import Call

pytestmark = pytest.mark.gpu


def backward_bounds(x):
    """Gradients in 64 bits, and what a kernel may be off by that forms D as the fp32 sum of P dP.  With A = |dO| |V|^T: dP is off by
    2^-16 A (128 products, added in fp32 with steps of 2^-23); S likewise by 2^-16 |scale| |Q| |K|^T, and with it lse, so P by t =
    2 * 2^-16 * that (the largest of the row) + 2^-18 relative to itself (exponential, sums, lse's own step of 2^-24 |lse| <= 2^-18); D then
    by sum P (2^-16 A + t |dP|); dS by its own rounding (2^-8), t, and P times the errors of dP and D."""
    s, qq, kk, dead, off = P.cross_parts(x.q, x.k, float(torch.tensor(x.scale, dtype=torch.float32)), x.q_lens, x.k_lens)
    G = x.q.shape[1] // x.k.shape[1]
    B, Hkv, Lk, d = x.k.shape
    vv = P.values(x.v, dead, G)
    do = torch.where(off[..., None], 0.0, x.dout.double())
    flip = lambda m: m.transpose(2, 3).contiguous()
    lse = torch.logsumexp(s, -1)
    p = torch.where(off[..., None], 0.0, torch.exp(s - lse[..., None]))
    dp, A = do @ flip(vv), do.abs() @ flip(vv.abs())
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    t = 2 * 2.0 ** -16 * x.scale * (qq.abs() @ flip(kk.abs())).amax(-1, keepdim=True) + 2.0 ** -18
    err = (2.0 ** -8 + t) * ds.abs() + p * (2.0 ** -16 * A + (p * (2.0 ** -16 * A + t * dp.abs())).sum(-1, keepdim=True))
    heads = lambda m: m.view(B, Hkv, G, Lk, d).sum(2)
    out = ((x.scale * (ds @ kk), x.scale * (err @ kk.abs())), (x.scale * heads(flip(ds) @ qq), x.scale * heads(flip(err) @ qq.abs())))
    # (a sum in fp32 of as many terms as rows or keys: 2^-16 of its size covers 128 of them)
    return [(g, b * (1 + 2.0 ** -8) + 2.0 ** -8 * g.abs() + 2.0 ** -16 * size + 2.0 ** -126)
            for (g, b), size in zip(out, (x.scale * (ds.abs() @ kk.abs()), x.scale * heads(flip(ds.abs()) @ qq.abs())))]


#     B  Hkv G  Lq  Lk    d    q_lens          k_lens
SHORT = [
    (3, 2, 1, 100, 128, 128, [100, 100, 100], [3, 77, 128]),
    (3, 2, 2, 60, 300, 128, [60, 60, 31], [3, 77, 128]),          # resident keys
    (3, 2, 1, 90, 512, 128, [90, 3, 90], [3, 77, 128]),           # rings or ranges of keys, by the padded length
    (3, 2, 1, 70, 4096, 128, [70, 70, 70], [3, 65, 128]),
    (3, 65, 1, 100, 512, 128, [100, 99, 100], [3, 77, 128]),      # rings
    (3, 65, 1, 100, 900, 64, [100, 99, 100], [2, 77, 128]),
    (3, 2, 2, 64, 900, 64, [64, 64, 64], [2, 77, 128]),
]


@pytest.mark.parametrize("shape", SHORT, ids=lambda s: "x".join(map(str, s[:6])))
def test_few_keys_in_a_padded_batch(shape):
    # softmaxes that are nearly one key (scores of size 4): dS = P (dP - D) nearly cancels, and D from the rounded result would show
    x = Call(*shape, gain=4.0)
    x.forward()
    ref = backward_bounds(x)
    x.out.fill_(math.nan)       # up to 128 keys the result is not read
    dq, dk, dv = x.backward()
    for name, got, (want, bound) in zip(("dq", "dk"), (dq, dk), ref):
        off = (got.double() - want).abs()
        bad = ~(off <= bound)
        assert int(bad.sum()) == 0, "%s: %d of %d off, worst %.3g of what is allowed" % (name, int(bad.sum()), bad.numel(), float((off / bound)[bad].max()))
        # root mean square, entry by entry: two roundings (dS, the result) of rms 0.41 * 2^-8 each (uniform over a binade), 0.0023
        # together; a third of that for all the rest
        for b in range(shape[0]):
            assert float((got[b].double() - want[b]).norm()) <= 0.003 * float(want[b].norm()), (name, b)
    assert dv.isfinite().all()


def test_entries_on_both_sides_of_128_keys():
    # the entry with 129 keys takes D from the result, its neighbours do not; each is what it is in a batch of its own
    shape = (3, 2, 1, 100, 400, 128, [100, 100, 100], [128, 129, 5])
    x = Call(*shape)
    x.forward()
    together = x.backward()
    for b in range(3):
        y = Call(*shape)
        for name in ("q", "k", "v", "dout", "q_lens", "k_lens", "out", "lse"):
            setattr(y, name, getattr(x, name)[b:b + 1].contiguous())
        for a, c in zip(together, y.backward()):
            assert ((a[b].double() - c[0].double()).abs() <= 2.0 ** -7 * c[0].double().abs() + 1e-5).all()
