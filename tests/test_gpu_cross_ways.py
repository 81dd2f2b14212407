"""Which way cross attention goes where sizes decide: few query rows for each of many key heads."""
import pytest
import torch

import plain_ops as P
from test_gpu_cross import Problem, near, within
from test_gpu_cross_turns import kernels_of

pytestmark = pytest.mark.gpu

#    B Hkv  G  Lq  Lk    d   storage scale q_lens k_lens        ranges in single waves, or a kernel of whole workgroups
CASES = [
    ((4, 40, 1, 1, 2049, 128, "blhd", None, None, [2049, 1000, 0, 1]), True),       # one token of many key heads
    ((2, 66, 5, 1, 1500, 128, "bhld", None, None, [1500, 333]), True),
    ((2, 70, 1, 64, 1100, 128, "blhd", None, [64, 33], None), True),                # two tiles to a key head
    ((2, 70, 1, 65, 1100, 128, "blhd", None, [65, 33], None), False),               # three
    ((1, 1300, 1, 1, 700, 64, "blhd", None, None, None), True),
    ((1, 270, 5, 31, 700, 64, "bhld", None, None, [641]), True),                    # five
    ((1, 240, 1, 161, 700, 64, "bhld", None, [161], [641]), False),                 # six
]


@pytest.mark.parametrize("case,single", CASES, ids=["-".join(map(str, c[0][:6])) for c in CASES])
def test_way(case, single):
    x = Problem(case, seed=71)
    (out, lse), names = kernels_of(x.forward)
    reached = [any(n.startswith(start % x.d) for n in names) for start in ("fgattn_fwd_kernel<32,%d,-1,", "cross_kernel<%d,")]
    assert reached == [single, not single], names
    ref, ref_lse, bound, off = x.plain(P.cross_forward)
    on = ~off
    within(out[on], ref[on], bound[on], "out")
    near(out[on], ref[on], "out")
    empty = ref_lse == -float("inf")
    assert (lse[on & empty] == -float("inf")).all() and (out[on & empty] == 0).all()
    assert ((lse.double() - ref_lse)[on & ~empty].abs() <= 2.0 ** -17 * (1 + ref_lse[on & ~empty].abs())).all()
