"""How head norms share a token's heads out over warps: by what fits on the SMs at once, and without a trace in the results."""
import os
import re

import pytest
import torch

from paper_2506_05096_b200 import binding as A

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_05096_b200", "csrc")


def test_shares_are_counted_by_the_warps_that_an_sm_holds():
    text = open(os.path.join(CSRC, "head_norm.cu")).read()
    assert re.search(r"__launch_bounds__\(kWarps \* 32, kBlocksSM\) head_norm_kernel", text)
    assert re.search(r"slots = \(long long\)sm_count\(\) \* \(kWarps \* kBlocksSM\);", text)
    assert re.search(r"static_assert\(kBlocksSM \* \(kSmem", text)


@pytest.mark.gpu
@pytest.mark.parametrize("d,H", [(64, 48), (72, 16), (72, 31), (128, 24), (128, 33)])
@pytest.mark.parametrize("norm", [A.NORM_RMS, A.NORM_LAYER])
def test_results_do_not_depend_on_the_shares(d, H, norm):
    """A row's result is the same alone, among few rows (its heads on several warps) and among many (all on one)."""
    g = torch.Generator("cuda").manual_seed(d + H)
    N = 6000
    x = torch.randn(1, N, H, d, device="cuda", generator=g).bfloat16()
    w, b = torch.randn(d, device="cuda", generator=g).bfloat16(), torch.randn(d, device="cuda", generator=g).bfloat16()
    angle = torch.randn(N, d // 2, device="cuda", generator=g)
    cos, sin = angle.cos(), angle.sin()
    st = A.bhnd_strides(N, H, d)

    def run(rows):
        y = torch.full_like(x, 7.0)
        idx = torch.arange(N, device="cuda", dtype=torch.int32)[None, N - rows:].contiguous()
        A.astraea_qk_norm_rotate([A.head_rows(x, st, y, st, H, idx, rows, w, b if norm == A.NORM_LAYER else None)], cos, sin, N, 1, N, d, norm=norm,
                                 rotation=A.ROTATE_HALF)
        assert bool((y[0, :N - rows] == 7).all())
        return y[0, N - rows:]

    whole = run(N)
    for rows in (1, 2, 149, 300, 394, 395, 473, 592, 789, 790, 1184, 1185, 2368, 2369, 4736, 4737):
        assert torch.equal(run(rows), whole[N - rows:]), rows
