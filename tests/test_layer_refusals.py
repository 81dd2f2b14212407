"""CPU-only: what the rotary and the cross attention calls refuse, before any device is touched, and the layout of their params."""
import ctypes
import os

import pytest
import torch

from paper_2509_16518_amd import build
from paper_2509_16518_amd import fgattn as F

AT = ctypes.c_void_p(4096)    # never dereferenced
ODD = ctypes.c_void_p(4100)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(build.LIBFGATTN):
        build.build_hip()
    return F.lib()


def rope_params(**change):
    B, Hq, Hk, L, d = 2, 4, 2, 100, 64
    p = F.FgattnRopeParams(B, Hq, Hk, L, d, 64, F.ROPE_INTERLEAVED, F.BF16, F.FLAG_ROPE_NORM, 1e-6, *(Hq * L * d, L * d, d), *(Hk * L * d, L * d, d),
                           *(Hq * L * d, L * d, d), *(Hk * L * d, L * d, d))
    for name, value in change.items():
        setattr(p, name, value)
    return p


def rope_forward(p, q=AT, k=AT, qw=AT, kw=AT, cos=AT, sin=AT, rows=100, positions=None, qo=AT, ko=AT):
    return F.lib().fgattn_rope_forward(q, k, qw, kw, cos, sin, rows, positions, None if p is None else ctypes.byref(p), qo, ko, None)


def rope_backward(p, q=AT, k=AT, qw=AT, kw=AT, gq=AT, gk=AT, dq=AT, dk=AT, dqw=AT, dkw=AT, ws=AT, nbytes=1 << 30):
    return F.lib().fgattn_rope_backward(q, k, qw, kw, AT, AT, 100, None, ctypes.byref(p), gq, gk, dq, dk, dqw, dkw, ws, nbytes, None)


def cross_params(**change):
    B, H, Hkv, Lq, Lk, d = 2, 4, 2, 300, 77, 128
    q, k = (H * Lq * d, Lq * d, d), (Hkv * Lk * d, Lk * d, d)
    p = F.FgattnCrossParams(B, H, Hkv, Lq, Lk, d, *q, *k, *k, *q, *q, *q, *k, *k, 0.1, 0)
    for name, value in change.items():
        setattr(p, name, value)
    return p


def cross_forward(p, q=AT, k=AT, v=AT, q_lens=None, k_lens=None, out=AT, lse=AT, ws=AT, nbytes=1 << 40):
    return F.lib().fgattn_cross_forward(q, k, v, q_lens, k_lens, None if p is None else ctypes.byref(p), out, lse, ws, nbytes, None)


def cross_backward(p, t=None, lse=AT, q_lens=None, k_lens=None, ws=AT, nbytes=1 << 40):
    a = dict.fromkeys(("q", "k", "v", "out", "dout", "dq", "dk", "dv"), AT)
    a.update(t or {})
    return F.lib().fgattn_cross_backward(a["q"], a["k"], a["v"], a["out"], lse, a["dout"], q_lens, k_lens, None if p is None else ctypes.byref(p),
                                         a["dq"], a["dk"], a["dv"], ws, nbytes, None)


def test_layout_of_the_params():
    # ints first, then 64-bit strides; the float and the flags end the struct
    assert ctypes.sizeof(F.FgattnRopeParams) == 40 + 12 * 8 and F.FgattnRopeParams.q_stride_b.offset == 40
    assert ctypes.sizeof(F.FgattnCrossParams) == 24 + 24 * 8 + 8 and F.FgattnCrossParams.scale.offset == 24 + 24 * 8
    assert ctypes.sizeof(F.FgattnRopeAxis) == 8 + 7 * 8
    assert "type" in F.fgattn_strerror(F.E_DTYPE)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), F.E_SHAPE), (dict(Hq=0), F.E_SHAPE), (dict(Hk=-1), F.E_SHAPE), (dict(L=0), F.E_SHAPE), (dict(L=2 ** 24 + 1), F.E_SHAPE),
    (dict(d=60), F.E_SHAPE), (dict(d=264), F.E_SHAPE), (dict(d=0), F.E_SHAPE), (dict(rot_dims=63), F.E_SHAPE), (dict(rot_dims=66), F.E_SHAPE),
    (dict(rot_dims=-2), F.E_SHAPE), (dict(layout=2), F.E_SHAPE), (dict(B=200, L=2 ** 24), F.E_SHAPE), (dict(Hq=70000), F.E_SHAPE),
    (dict(dtype=3), F.E_DTYPE), (dict(dtype=-1), F.E_DTYPE), (dict(flags=4), F.E_FLAGS), (dict(eps=float("nan")), F.E_SCALE),
    (dict(eps=float("inf")), F.E_SCALE), (dict(eps=-1e-6), F.E_SCALE), (dict(q_stride_l=65), F.E_STRIDE), (dict(k_stride_h=-64), F.E_STRIDE),
    (dict(qo_stride_l=56), F.E_STRIDE), (dict(ko_stride_b=0), F.E_STRIDE), (dict(qo_stride_h=0), F.E_STRIDE)])
def test_rope_params(change, code):
    assert rope_forward(rope_params(**change)) == code
    if code in (F.E_SHAPE, F.E_DTYPE, F.E_FLAGS, F.E_SCALE):
        assert F.fgattn_rope_workspace_bytes(rope_params(**change)) == 0


def test_rope_arguments():
    p = rope_params()
    assert rope_forward(None) == F.E_NULL
    for missing in ("q", "k", "cos", "sin", "qo", "ko"):
        assert rope_forward(p, **{missing: None}) == F.E_NULL, missing
    for odd in ("q", "k", "qo", "ko"):
        assert rope_forward(p, **{odd: ODD}) == F.E_ALIGN, odd
    for odd in ("qw", "kw", "cos", "sin", "positions"):
        assert rope_forward(p, **{odd: ctypes.c_void_p(4097)}) == F.E_ALIGN, odd
    assert rope_forward(rope_params(flags=3), qw=ctypes.c_void_p(4098)) == F.E_ALIGN       # fp32 weights
    assert rope_forward(p, rows=99) == F.E_SHAPE                                           # token 99 has no row
    assert rope_forward(p, rows=0, positions=AT) == F.E_SHAPE
    assert rope_forward(rope_params(flags=0)) == F.E_FLAGS                                 # weights without the norm
    assert rope_forward(rope_params(Hk=0), kw=AT) == F.E_SHAPE
    # what is read may be broadcast, what is written may not: backward, the strides of q are its gradient's
    assert rope_backward(rope_params(q_stride_b=0)) == F.E_STRIDE
    assert rope_backward(p, gq=None) == F.E_NULL and rope_backward(p, dk=None) == F.E_NULL and rope_backward(p, q=None) == F.E_NULL
    assert rope_backward(p, gk=ODD) == F.E_ALIGN and rope_backward(p, dqw=ctypes.c_void_p(4098)) == F.E_ALIGN
    assert rope_backward(p, ws=None) == F.E_NULL and rope_backward(p, ws=ODD) == F.E_ALIGN
    assert rope_backward(p, nbytes=F.fgattn_rope_workspace_bytes(p) - 1) == F.E_WORKSPACE
    assert rope_backward(rope_params(flags=0), qw=None, kw=None) == F.E_FLAGS              # weight gradients without the norm


def axis(**change):
    x = F.FgattnRopeAxis(10, 8, 10000.0, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0)
    for name, value in change.items():
        setattr(x, name, value)
    return x


def table(*axes, mscale=1.0, cos=AT, sin=AT):
    return F.lib().fgattn_rope_table((F.FgattnRopeAxis * max(1, len(axes)))(*axes), len(axes), mscale, cos, sin, None)


def test_rope_table_arguments():
    inf, nan = float("inf"), float("nan")
    assert F.lib().fgattn_rope_table(None, 1, 1.0, AT, AT, None) == F.E_NULL
    assert table(axis(), cos=None) == F.E_NULL and table(axis(), sin=None) == F.E_NULL
    assert table() == F.E_SHAPE and table(*[axis()] * 4) == F.E_SHAPE
    for bad in (dict(size=0), dict(size=2 ** 24 + 1), dict(pairs=0), dict(pairs=129)):
        assert table(axis(**bad)) == F.E_SHAPE, bad
    assert table(axis(size=2 ** 13), axis(size=2 ** 12)) == F.E_SHAPE and table(axis(pairs=100), axis(pairs=29)) == F.E_SHAPE
    for bad in (dict(theta=0.0), dict(theta=-2.0), dict(theta=nan), dict(offset=inf), dict(step=nan), dict(factor=0.0), dict(factor=inf),
                dict(original=-1.0), dict(original=nan), dict(original=10.0, beta_fast=1.0), dict(original=10.0, beta_slow=nan)):
        assert table(axis(), axis(**bad)) == F.E_SCALE, bad
    assert table(axis(), mscale=nan) == F.E_SCALE
    assert table(axis(), cos=ctypes.c_void_p(4097)) == F.E_ALIGN
    with pytest.raises(F.FgattnError):
        F.fgattn_rope_table([], torch.empty(1), torch.empty(1))


@pytest.mark.parametrize("change,code", [
    (dict(B=0), F.E_SHAPE), (dict(H=0), F.E_SHAPE), (dict(Hkv=0), F.E_SHAPE), (dict(Hkv=3), F.E_SHAPE), (dict(Lq=0), F.E_SHAPE), (dict(Lk=0), F.E_SHAPE),
    (dict(Lq=2 ** 24 + 1), F.E_SHAPE), (dict(Lk=2 ** 24 + 1), F.E_SHAPE), (dict(d=96), F.E_SHAPE), (dict(H=2 ** 10, Hkv=1, Lq=2 ** 22), F.E_SHAPE),
    (dict(B=2 ** 20, H=2 ** 10, Hkv=2 ** 10), F.E_SHAPE), (dict(flags=1), F.E_FLAGS), (dict(scale=float("nan")), F.E_SCALE), (dict(scale=float("-inf")), F.E_SCALE),
    (dict(q_stride_l=100), F.E_STRIDE), (dict(k_stride_l=132), F.E_STRIDE), (dict(v_stride_b=-8), F.E_STRIDE),
    (dict(k_stride_l=2 ** 23), F.E_STRIDE)])
def test_cross_params(change, code):
    assert cross_forward(cross_params(**change)) == code
    assert cross_backward(cross_params(**change)) == code
    if code in (F.E_SHAPE, F.E_FLAGS, F.E_SCALE):
        assert F.fgattn_cross_workspace_bytes(cross_params(**change)) == 0 == F.fgattn_cross_backward_workspace_bytes(cross_params(**change))


def test_cross_arguments():
    p = cross_params()
    assert cross_forward(None) == F.E_NULL and cross_backward(None) == F.E_NULL
    for missing in ("q", "k", "v", "out", "lse"):
        assert cross_forward(p, **{missing: None}) == F.E_NULL, missing
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        assert cross_backward(p, {name: None}) == F.E_NULL and cross_backward(p, {name: ODD}) == F.E_ALIGN, name
    for odd in ("q", "k", "v", "out"):
        assert cross_forward(p, **{odd: ODD}) == F.E_ALIGN, odd
    assert cross_forward(p, lse=ctypes.c_void_p(4097)) == F.E_ALIGN and cross_forward(p, k_lens=ctypes.c_void_p(4098)) == F.E_ALIGN
    assert cross_forward(cross_params(o_stride_h=0)) == F.E_STRIDE
    for name in ("dq", "dk", "dv"):      # gradients are written: no broadcast dimension
        assert cross_backward(cross_params(**{name + "_stride_h": 0})) == F.E_STRIDE
    assert cross_backward(p, lse=None) == F.E_NULL and cross_backward(p, q_lens=ctypes.c_void_p(4097)) == F.E_ALIGN
    need = F.fgattn_cross_backward_workspace_bytes(p)
    assert need > 0 and cross_backward(p, nbytes=need - 1) == F.E_WORKSPACE and cross_backward(p, ws=None) == F.E_NULL and cross_backward(p, ws=ODD) == F.E_ALIGN
    few = cross_params(Lq=1, Lk=9000, k_stride_h=9000 * 128, k_stride_b=2 * 9000 * 128, v_stride_h=9000 * 128, v_stride_b=2 * 9000 * 128)
    need = F.fgattn_cross_workspace_bytes(few)
    assert need > 0 and cross_forward(few, nbytes=need - 1) == F.E_WORKSPACE and cross_forward(few, ws=None) == F.E_NULL
    # slices that 32-bit offsets do not reach (4096 steps of 1 MiB are 4 GiB): keys and values always, queries and their gradient's source in the backward call
    far = dict(Lk=2 ** 12 + 1, k_stride_l=2 ** 19)
    assert cross_forward(cross_params(**far)) == F.E_STRIDE
    assert cross_backward(cross_params(Lq=2 ** 12 + 1, q_stride_l=2 ** 19)) == F.E_STRIDE
    assert cross_backward(cross_params(Lq=2 ** 12 + 1, do_stride_l=2 ** 19)) == F.E_STRIDE


def expect(code, call):
    with pytest.raises(F.FgattnError) as e:
        call()
    assert e.value.code == code


def test_bindings_compare_tensors_with_the_params():
    q, k = torch.zeros(2, 4, 9, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 9, 64, dtype=torch.bfloat16)
    cos = torch.zeros(9, 32)
    p = F.make_rope_params(q, k, q, k, 64)
    call = lambda qq=q, kk=k, c=cos, s=cos, **more: F.fgattn_rope_forward(qq, kk, p, q, k, c, s, **more)
    expect(F.E_DEVICE, call)                                    # (host tensors, once everything else is right)
    expect(F.E_DTYPE, lambda: call(qq=q.half()))
    expect(F.E_SHAPE, lambda: call(qq=q[:, :, :8]))
    expect(F.E_STRIDE, lambda: call(qq=torch.zeros(2, 9, 4, 64, dtype=torch.bfloat16).transpose(1, 2)))
    expect(F.E_SHAPE, lambda: call(c=torch.zeros(9, 64)))
    expect(F.E_SHAPE, lambda: call(c=torch.zeros(32, 9).t()))
    expect(F.E_DTYPE, lambda: call(c=cos.double()))
    expect(F.E_NULL, lambda: call(c=None))
    expect(F.E_DTYPE, lambda: call(positions=torch.zeros(2, 9, dtype=torch.int64)))
    expect(F.E_SHAPE, lambda: call(positions=torch.zeros(9, dtype=torch.int32)))
    expect(F.E_DTYPE, lambda: call(q_weight=torch.zeros(64)))
    expect(F.E_SHAPE, lambda: call(q_weight=torch.zeros(32, dtype=torch.bfloat16)))
    expect(F.E_DTYPE, lambda: F.make_rope_params(q.double(), k, q, k, 64))
    expect(F.E_SHAPE, lambda: F.make_rope_params(q, k[:, :, :8], q, k[:, :, :8], 64))
    expect(F.E_SHAPE, lambda: F.make_rope_params(q, k, q, None, 64))
    expect(F.E_STRIDE, lambda: F.make_rope_params(q.transpose(2, 3), None, q.transpose(2, 3), None, 8))
    expect(F.E_SHAPE, lambda: F.fgattn_rope_table([(9, 16, 10000.0)], cos, cos))
    kv, lse = torch.zeros(2, 2, 5, 64, dtype=torch.bfloat16), torch.zeros(2, 4, 9)
    p2 = F.make_cross_params(q, kv, kv, q, 0.1)
    cross = lambda kk=kv, l=lse, **more: F.fgattn_cross_forward(q, kk, kv, p2, q, l, **more)
    expect(F.E_DEVICE, cross)
    expect(F.E_DTYPE, lambda: cross(kk=kv.half()))
    expect(F.E_SHAPE, lambda: cross(kk=kv[:, :, :4]))
    expect(F.E_SHAPE, lambda: cross(l=torch.zeros(2, 4, 8)))
    expect(F.E_SHAPE, lambda: cross(k_lens=torch.zeros(3, dtype=torch.int32)))
    expect(F.E_DTYPE, lambda: cross(q_lens=torch.zeros(2)))
    expect(F.E_SHAPE, lambda: F.make_cross_params(q, kv, kv[:, :, :4], q, 0.1))
    expect(F.E_STRIDE, lambda: F.make_cross_params(q, kv.transpose(2, 3).contiguous().transpose(2, 3), kv, q, 0.1))


def test_bindings_refuse_what_the_pointers_would_hide():
    # an axis without its theta, or with more than an axis has
    out = torch.zeros(9, 32)
    expect(F.E_SHAPE, lambda: F.fgattn_rope_table([(9, 32)], out, out))
    expect(F.E_SHAPE, lambda: F.fgattn_rope_table([(9, 32, 1e4, 0.0, 1.0, 1.0, 0.0, 32.0, 1.0, 1.0)], out, out))
    # a table of 2^32 + 9 rows, which 32 bits would take for 9 (no memory behind it)
    q = torch.zeros(1, 2, 9, 64, dtype=torch.bfloat16)
    p = F.make_rope_params(q, None, q, None, 64)
    many = torch.empty(2 ** 32 + 9, 32, device="meta")
    expect(F.E_SHAPE, lambda: F.fgattn_rope_forward(q, None, p, q, None, many, many))
    # a workspace of one element seen a million times
    kv, lse = torch.zeros(1, 1, 9000, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 9)
    p = F.make_cross_params(q, kv, kv, q, 0.1, q, q, kv, kv)
    thin = torch.zeros(1, dtype=torch.uint8).expand(F.fgattn_cross_backward_workspace_bytes(p))
    expect(F.E_SHAPE, lambda: F.fgattn_cross_forward(q, kv, kv, p, q, lse, thin))
    expect(F.E_SHAPE, lambda: F.fgattn_cross_backward(q, kv, kv, q, lse, q, p, q, kv, kv, thin))
    w = torch.zeros(64, dtype=torch.float32)
    p = F.make_rope_params(q, None, q, None, 0)
    thin = torch.zeros(1, dtype=torch.uint8).expand(F.fgattn_rope_workspace_bytes(p))
    expect(F.E_SHAPE, lambda: F.fgattn_rope_backward(q, None, p, q, None, q, None, dq_weight=w, workspace=thin))


def test_rope_tokens_stay_within_a_launch():
    # 2^25 tokens of the widest rows are 2^23 workgroups of 256 threads
    assert F.fgattn_rope_workspace_bytes(rope_params(L=2 ** 24)) > 0                  # (two batch entries)
    assert F.fgattn_rope_workspace_bytes(rope_params(B=3, L=2 ** 24)) == 0
    assert rope_forward(rope_params(B=3, L=2 ** 24), rows=2 ** 24) == F.E_SHAPE
