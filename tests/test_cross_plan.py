"""Cross attention's ranges of keys, as the workspace tells them: what the kernels that are built rely on."""
import math
import random

from paper_2509_16518_amd import fgattn as F


def ranges(B, Hkv, G, Lq, Lk, d):
    """(32-row tiles of a key head, how many ranges a forward call splits its keys into, by its workspace)"""
    s = d * max(Lq, Lk)
    p = F.FgattnCrossParams(B=B, H=Hkv * G, Hkv=Hkv, Lq=Lq, Lk=Lk, d=d, scale=0.1, **{"%s_stride_%s" % (t, x): v for t in ("q", "k", "v", "o")
                                                                                      for x, v in (("b", s * Hkv * G), ("h", s), ("l", d))})
    tiles = -(-G * Lq // 32)
    part = B * Hkv * tiles * 32 * (d + 2) * 4
    size = F.fgattn_cross_workspace_bytes(p)
    return tiles, size // part if size else 1


def test_ranges_of_small_heads_hold_more_keys_than_lds():
    # d = 64, enough tiles for whole workgroups: one range, or two of more than 640 keys each (no kernel joins parts of resident keys)
    rng, split = random.Random(5), 0
    size = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    for _ in range(20000):
        B, Hkv, G, Lq, Lk = size(1, 8), size(1, 60), size(1, 8), size(100, 60000), size(641, 100000)
        tiles, n = ranges(B, Hkv, G, Lq, Lk, 64)
        if tiles < 6 or B * Hkv * tiles < 1280:
            continue
        split += n > 1
        assert n == 1 or (n == 2 and -(-Lk // 2) > 640)
    assert split > 10
    assert ranges(1, 1, 1, 41600, 2100, 64)[1] == 2 and ranges(1, 1, 1, 41600, 2000, 64)[1] == 1
