"""Operators on 8-bit floats on an MI355X where their numbers are far from ordinary: sums that cancel, gates and scales at the ends of
their range, sizes that take several launches."""
import numpy as np
import pytest
import torch

import fp8_util as U

pytestmark = pytest.mark.gpu

q = pytest.importorskip("paper_2111_09547_amd")

# one size for each kernel of the products: few rows, tiles of 128 x 128, tiles of 256 x 256
SIZES = [(3, 128, 128), (300, 2050, 2050), (4090, 4090, 1100)]


def on_device(m):
    """What a matrix in 8-bit floats holds, fp32."""
    return (m.codes.float() * m.scales[:, :m.blocks].float().repeat_interleave(128, 1))[:, :m.cols]


@pytest.mark.parametrize("rows,cols,inner", SIZES)
@pytest.mark.parametrize("groups,small", [(1, -5), (2, -6), (4, -7), (1, -1), (1, 7), (4, 7)])
def test_gated_scale_where_sums_cancel(rows, cols, inner, groups, small):
    """Column 0's gate is 448^2 - 448^2 + 6 small in each of some groups of 8 products, and 56: the 8-bit instruction cuts the small ones
    off, and h = 56 * 8 lies on a border between two scales.  Computed again it is anything up to 98 * 8.  Whatever column 0 becomes
    between the two (silu is monotonous from -1 on and within 0.3 of 0 below), the other columns' sums are exact: 52 * 8."""
    x, g, u = torch.zeros((rows, inner)), torch.zeros((cols, inner)), torch.zeros((cols, inner))
    for k in range(0, 8 * groups, 8):
        x[:, k:k + 2], x[:, k + 2:k + 8] = 448.0, 1.0
        g[0, k], g[0, k + 1], g[0, k + 2:k + 8] = 448.0, -448.0, float(small)
    x[:, 120:122] = 1.0
    g[0, 120], g[1:, 120], g[1:, 100] = 56.0, 52.0, 448.0        # (scales are 1: no code is rounded)
    u[:, 121], u[:, 101] = 8.0, 448.0
    X, G, P = (q.qgtc_fp8_quantize(t.cuda()) for t in (x, g, u))
    got = on_device(q.qgtc_fp8_gated(X, G, P))
    exact = 56.0 + 6 * small * groups
    lo, hi = 8 * min(56.0, max(exact, -0.3)), 8 * max(56.0, exact)
    assert bool((got[:, 1:] == 416.0).all())                     # (13 * 32: an e4m3)
    assert bool((got[:, 0] >= lo * (1 + 2.0 ** -4 * np.sign(-lo))).all() and (got[:, 0] <= hi * (1 + 2.0 ** -4)).all()), got[:2, 0].tolist()
