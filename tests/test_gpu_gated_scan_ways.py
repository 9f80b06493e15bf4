"""Every way in which the gated scan deals its runs, in its steady state: each warp's ring refilled several times, each place of a chain handed
over more than twice, several rounds of a cluster.  The way taken is asked for, so that a size cannot quietly test another one.  References and
tolerances are those of test_gpu_gated_scan.py."""
import pytest

from paper_2312_17530_b200 import binding
from test_gpu_gated_scan import call

pytestmark = pytest.mark.gpu
ONE = (1,)


@pytest.mark.parametrize("kind,layout", [("bf16", "batch"), ("f16", "odd"), ("f32", "batch"), ("f32", "odd")])
@pytest.mark.parametrize("n,t,d,short,single", [
    # sizes; (warps, CTAs) forward and backward in 16-bit types, in binary32
    (1300, 200, 64, ((1, ONE), (1, ONE)), ((1, ONE), (1, ONE))),
    (700, 300, 64, ((2, ONE), (1, ONE)), ((2, ONE), (1, ONE))),
    (500, 300, 64, ((4, ONE), (2, ONE)), ((2, ONE), (2, ONE))),
    (250, 700, 64, ((8, ONE), (4, ONE)), ((4, ONE), (4, ONE))),
    (200, 700, 64, ((8, ONE), (4, ONE)), ((8, ONE), (4, ONE))),
    (140, 700, 64, ((12, ONE), (12, ONE)), ((12, ONE), (8, ONE))),
    (140, 175, 64, ((8, ONE), (8, ONE)), ((8, ONE), (8, ONE))),
    # two CTAs; forward not in binary32.  In the backward pass 16 warps of each take aligned rows of 16-bit types, 12 others
    (7, 1100, 520, ((16, (2,)), (0, (2,))), ((12, ONE), (8, (2,)))),
    (1, 2100, 64, ((16, (4,)), (0, (4, 5))), ((8, (8,)), (8, (8,)))),
    # 17 groups: eight CTAs each, or as many as the device holds of all of them at a time
    (1, 4200, 1032, ((16, (6, 7, 8)), (0, (6, 7, 8))), ((8, (6, 7, 8)), (8, (6, 7, 8))))])
def test_ways(monkeypatch, n, t, d, short, single, kind, layout):
    taken = []
    for name in ("gated_scan_forward", "gated_scan_backward"):
        def recorded(*args, _call=getattr(binding, name)):
            _call(*args)
            taken.append(binding.selftest_scan_way())
        monkeypatch.setattr(binding, name, recorded)
    call(n, t, d, kind, layout, restart=0.01, ragged=n > 1)
    split = 8 if kind == "f32" else 16 if layout == "batch" else 12
    for (warps, ctas), (want_warps, want_ctas) in zip(taken, single if kind == "f32" else short):
        assert warps == (want_warps or split) and ctas in want_ctas, taken
