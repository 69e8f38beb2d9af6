"""The layer on 4-bit operands with more tiles than one launch holds."""
import os
import re

import pytest
import torch

import paper_2505_20932_amd as P
from oracle import mx4_oracle as mx

DEV = "cuda:0"
_RULES = os.path.join(os.path.dirname(P.__file__), "csrc", "mx4_rules.h")


def test_a_launch_counts_fewer_than_2_to_the_32_threads():
    at = re.search(r"kMx4TilesPerLaunch = \(\(int64_t\)1 << (\d+)\) / (\d+);", open(_RULES).read())
    assert 2 ** int(at.group(1)) // int(at.group(2)) * 256 < 2 ** 32


@pytest.mark.gpu
def test_2_to_the_29_rows():
    """2^24 + 2 tiles of 32 x 32: rows around the borders of the launches, the first and the last."""
    m, n, k = 2 ** 29 + 37, 3, 32
    print(f"{m} x {n} x {k}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(4)
    xc = torch.randint(0, 256, (m, k // 2), dtype=torch.uint8, device=DEV, generator=g)
    xs = torch.zeros(1, m, 8, dtype=torch.uint8, device=DEV)
    xs[0, :, 0] = 127
    wc = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device=DEV, generator=g)
    ws = torch.zeros(1, n, 8, dtype=torch.uint8, device=DEV)
    ws[0, :, 0] = 126
    out = torch.full((m + 1, n), -777.0, dtype=torch.float16, device=DEV)
    P.qlinear_mx4_cwac_forward(xc, xs, wc, ws, None, None, out[:m])
    torch.cuda.synchronize()
    assert (out[m] == -777).all()
    w = mx.values(mx.unpack(wc.cpu().numpy()), ws[0, :, :1].cpu().numpy())
    for at in (0, 2 ** 28 - 500, 2 ** 29 - 500, m - 1000):
        rows = slice(at, min(at + 1000, m))
        x = mx.values(mx.unpack(xc[rows].cpu().numpy()), xs[0, rows, :1].cpu().numpy())
        want = torch.from_numpy(x @ w.T)                             # quarters below 2^9: exact in fp32, rounded once
        assert torch.equal(out[rows].cpu(), want.half())
    assert int((out[:m] == -777).sum()) == 0                          # no row is left out
