"""What lies in query rows behind their sequences does not reach the counted rows, not even their last bit."""
import math

import pytest
import torch

from test_gpu_cross import Problem
from test_gpu_cross_turns import kernels_of

pytestmark = pytest.mark.gpu

#    B Hkv G  Lq    Lk   d   storage scale  q_lens         k_lens      a kernel that the call reaches
CASES = [
    ((2, 12, 1, 500, 226, 128, "blhd", None, [473, 7], [226, 90]), "cross_kernel<128,8,false,false>"),
    ((2, 6, 2, 500, 333, 64, "bhld", None, [500, 7], None), "cross_kernel<64,12,false,false>"),
    ((2, 12, 2, 500, 700, 128, "bhld", None, [473, 7], [700, 65]), "cross_kernel<128,8,true,false>"),
    ((2, 24, 1, 1000, 700, 64, "blhd", None, [977, 7], None), "cross_kernel<64,8,true,false>"),
    ((1, 1, 1, 4000, 2000, 128, "bhld", None, [3977], None), "cross_kernel<128,8,false,true>"),
    ((1, 12, 1, 1000, 2048, 128, "bhld", None, [977], None), "cross_kernel<128,8,true,true>"),
    ((3, 2, 8, 1, 1031, 64, "blhd", None, [1, 0, 1], [1031, 128, 1]), "join_kernel<64>"),
    ((2, 4, 5, 3, 8191, 128, "bhld", None, [1, 2], [8191, 17]), "join_kernel<128>"),
    ((2, 3, 2, 45, 97, 128, "blhd", None, [44, 3], [97, 90]), "fgattn_fwd_kernel<32,128,-1"),
]


@pytest.mark.parametrize("case,kernel", CASES, ids=["-".join(map(str, c[0][:6])) for c in CASES])
def test_rows_behind_the_sequences(case, kernel):
    x = Problem(case, seed=81, gain=2.0)
    gen = torch.Generator(device="cuda").manual_seed(82)
    found = []
    for what in (0.0, 4.0, 1e3, math.nan, math.inf):
        for b, n in enumerate(case[8]):
            rows = x.q[b, :, n:]
            rows.copy_(what * torch.randn(rows.shape, generator=gen, device="cuda"))
        x.out.fill_(99.0)
        x.lse.fill_(99.0)
        (out, lse), names = kernels_of(x.forward)
        reached = any(n.startswith(kernel) for n in names)
        assert reached, names
        found.append((out.clone(), lse.clone()))
    assert found[0][0].isfinite().all()
    for out, lse in found[1:]:
        changed = int((out != found[0][0]).sum()), int((lse != found[0][1]).sum())
        assert changed == (0, 0), changed
