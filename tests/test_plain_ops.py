"""The plain 64-bit definitions that the GPU tests compare with: gradients against differences, rotation against complex numbers."""
import math

import torch

import plain_ops as P


def difference(f, x, direction, h=1e-6):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def draw(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float64)


def test_rotation_is_a_product_with_a_complex_number():
    gen = torch.Generator().manual_seed(1)
    d, rot, L = 12, 8, 5
    cos, sin, angle = P.table([(L, rot // 2, 100.0, 3.0, 0.5, 1.0, 0.0, 32.0, 1.0)])
    x = draw(gen, 2, 3, L, d)
    for half in (False, True):
        y, _ = P.rope_forward(x.float(), None, P.turn_matrix(cos, sin, None, d, rot, half, L), 0.0, False)
        a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if half else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(x.float().double()[..., a], x.float().double()[..., b]) * torch.exp(1j * angle)
        assert torch.allclose(y[..., a], z.real, atol=1e-12) and torch.allclose(y[..., b], z.imag, atol=1e-12)
        assert torch.equal(y[..., rot:], x.float().double()[..., rot:])


def test_table_scaling_limits():
    plain = P.table([(50, 8, 10000.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0)])[2]
    linear = P.table([(50, 8, 10000.0, 0.0, 1.0, 4.0, 0.0, 32.0, 1.0)])[2]
    assert torch.allclose(linear, plain / 4)
    by_parts = P.table([(50, 8, 10000.0, 0.0, 1.0, 4.0, 1024.0, 32.0, 1.0)])[2]
    assert torch.allclose(by_parts[:, 0], plain[:, 0])            # 163 turns over the trained length: as it was
    assert torch.allclose(by_parts[:, -1], plain[:, -1] / 4)      # less than one: as slow as by interpolation
    assert torch.allclose(P.table([(50, 8, 10000.0, 0.0, 1.0, 4.0, 1024.0, 32.0, 1.0)], 1.5)[0], 1.5 * by_parts.cos())


def test_rope_gradients_against_differences():
    gen = torch.Generator().manual_seed(2)
    B, H, L, d, rot = 2, 2, 3, 10, 6
    cos, sin, _ = P.table([(L, rot // 2, 30.0, 1.0, 1.0, 1.0, 0.0, 32.0, 1.0)], 1.25)
    P_types = P.HALF, P.TINY
    for m in P_types:
        m.setdefault(torch.float64, 0.0)
    x, w, dy = draw(gen, B, H, L, d), 1 + 0.3 * draw(gen, d), draw(gen, B, H, L, d)
    for half in (False, True):
        R = P.turn_matrix(cos, sin, None, d, rot, half, L)
        for norm in (False, True):
            dx, _, dw, _ = P.rope_backward(x, w if norm else None, R, 1e-3, norm, dy)
            f = lambda xx, ww=w: (P.rope_forward(xx, ww if norm else None, R, 1e-3, norm)[0] * dy).sum()
            for _ in range(3):
                t = draw(gen, B, H, L, d)
                assert math.isclose(float((dx * t).sum()), float(difference(f, x, t)), rel_tol=1e-6, abs_tol=1e-6)
            if norm:
                t = draw(gen, d)
                assert math.isclose(float((dw * t).sum()), float(difference(lambda ww: f(x, ww), w, t)), rel_tol=1e-6, abs_tol=1e-6)


def test_cross_gradients_against_differences():
    gen = torch.Generator().manual_seed(3)
    B, H, Hkv, Lq, Lk, d = 3, 4, 2, 5, 7, 6
    q, k, v, dout = draw(gen, B, H, Lq, d), draw(gen, B, Hkv, Lk, d), draw(gen, B, Hkv, Lk, d), draw(gen, B, H, Lq, d)
    for q_lens, k_lens in ((None, None), (torch.tensor([5, 2, 0]), torch.tensor([7, 0, 3]))):
        grads = [g for g, _ in P.cross_backward(q, k, v, -0.7, dout, q_lens, k_lens)]

        def f(which, x):
            t = [q, k, v]
            t[which] = x
            out, _, _, off = P.cross_forward(*t, -0.7, q_lens, k_lens)
            return torch.where(off[..., None], 0.0, out * dout).sum()
        for which, x in enumerate((q, k, v)):
            for _ in range(3):
                t = draw(gen, *x.shape)
                assert math.isclose(float((grads[which] * t).sum()), float(difference(lambda y: f(which, y), x, t)), rel_tol=1e-6, abs_tol=1e-6)


def test_cross_forward_is_softmax_over_the_first_keys():
    gen = torch.Generator().manual_seed(4)
    q, k, v = draw(gen, 2, 2, 3, 4), draw(gen, 2, 1, 6, 4), draw(gen, 2, 1, 6, 4)
    k[1, :, 4:], v[1, :, 4:] = math.nan, math.inf
    out, lse, _, _ = P.cross_forward(q, k, v, 0.5, None, torch.tensor([0, 4]))
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    ref = torch.nn.functional.scaled_dot_product_attention(q[1:], k[1:, :, :4].expand(1, 2, 4, 4), v[1:, :, :4].expand(1, 2, 4, 4), scale=0.5)
    assert torch.allclose(out[1:], ref, atol=1e-12)
