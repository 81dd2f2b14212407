"""Cross attention where a workgroup goes through several query tiles per wave and several key heads: every kernel of the large
calls, resident keys and rings, in one range of keys and in several.  Each case names the kernels that it has to reach."""
import re

import pytest
import torch

import plain_ops as P
from test_gpu_cross import Problem, near, within

pytestmark = pytest.mark.gpu


def kernels_of(call):
    """Names of this library's kernels that a call launches, with their template arguments."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        result = call()
        torch.cuda.synchronize()
    found = set()
    for e in prof.events():
        m = re.search(r"\bfg\w?::(\w+(?:<[^>]*>)?)\(", e.name)
        if m:
            found.add(m.group(1).replace(" ", ""))
    return result, found


#    B Hkv G  Lq     Lk    d   storage scale  q_lens          k_lens     forward                        backward
CASES = [
    # rings, three tiles of a wave and more, ranges of a workgroup that end one key head and begin another; an entry with fewer keys than
    # the ring holds, whose tiles come round again within it
    ((2, 3, 1, 33000, 350, 128, "bhld", None, [33000, 32989], [350, 40]), {"cross_kernel<128,8,true,false>"}, {"dq_kernel<128,true>", "dkdv_kernel<128>"}),
    ((2, 3, 1, 33000, 700, 64, "blhd", None, [32990, 33000], [69, 700]), {"cross_kernel<64,8,true,false>"}, {"dq_kernel<64,true>", "dkdv_kernel<64>"}),
    # the same with query heads below each other, and a middle entry without keys
    ((3, 1, 5, 6700, 449, 128, "slice", 0.05, [6700, 6700, 411], [449, 0, 330]), {"cross_kernel<128,8,true,false>"}, {"dq_kernel<128,true>"}),
    # resident keys
    ((2, 3, 1, 33000, 333, 64, "blhd", None, [33000, 21001], [333, 1]), {"cross_kernel<64,12,false,false>"}, {"dq_kernel<64,false>"}),
    ((2, 3, 1, 33000, 200, 128, "bhld", None, [32001, 33000], [200, 65]), {"cross_kernel<128,8,false,false>"}, {"dq_kernel<128,false>"}),
    # ranges of keys: joined parts of resident keys, of rings
    ((1, 1, 1, 4000, 2000, 128, "blhd", None, [3999], [1997]), {"cross_kernel<128,8,false,true>", "join_few_kernel<128,8>"}, {"dq_kernel<128,false>", "sum_q_kernel<128>", "sum_kernel<128>"}),
    ((1, 24, 1, 511, 2048, 128, "bhld", None, None, [1500]), {"cross_kernel<128,8,true,true>", "join_few_kernel<128,8>"}, {"dq_kernel<128,true>", "sum_q_kernel<128>"}),
    ((1, 1, 1, 41600, 2100, 64, "bhld", None, [41590], [2099]), {"cross_kernel<64,8,true,true>", "join_few_kernel<64,2>"}, {"dq_kernel<64,true>"}),
]


@pytest.mark.parametrize("case,forward,backward", CASES, ids=["-".join(map(str, c[0][:7])) for c in CASES])
def test_turns(case, forward, backward):
    x = Problem(case, seed=51)
    (out, lse), names = kernels_of(x.forward)
    assert forward <= names, names
    ref, ref_lse, bound, off = x.plain(P.cross_forward)
    assert (out[off] == 99).all() and (lse[off] == 99).all()
    on = ~off
    within(out[on], ref[on], bound[on], "out")
    near(out[on], ref[on], "out")
    empty = ref_lse == -float("inf")
    assert (lse[on & empty] == -float("inf")).all() and (out[on & empty] == 0).all()
    assert ((lse.double() - ref_lse)[on & ~empty].abs() <= 2.0 ** -17 * (1 + ref_lse[on & ~empty].abs())).all()
    first = out.clone(), lse.clone()
    x.forward()
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    del ref, ref_lse, bound

    got, names = kernels_of(x.backward)
    assert backward <= names, names
    for name, g, (r, bound) in zip(("dq", "dk", "dv"), got, x.plain(P.cross_backward, x.dout)):
        within(g, r, bound, name)
        near(g, r, name, 2.0 ** -7)
    for a, b in zip(got, x.backward()):
        assert torch.equal(a, b)
