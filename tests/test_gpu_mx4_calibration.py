"""The layer on 4-bit operands calibrated: fp32 calibration forward, statistics, fit, fold, compensated forward, each step against its definition
on the output of the step before."""
import numpy as np
import pytest
import torch

import paper_2505_20932_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def _mx4(x):
    rows, k = x.shape
    codes = torch.empty(rows, k // 2, dtype=torch.uint8, device=DEV)
    scales = torch.empty(-(-k // 256), rows, 8, dtype=torch.uint8, device=DEV)
    P.cwac_mx4_quantize(x, codes, scales)
    v = torch.empty(rows, k, device=DEV)
    P.cwac_mx4_dequantize(codes, scales, v)
    return codes, scales, v.double()


def _bound(k, y, mag, t):
    """The output's rounding; the fp32 sums over K (a step of 2^-23 per 64 products), the join of partial ones and the epilogue's two operations."""
    return EPS[t] * y.abs() * (1 + 2.0 ** -10) + (k / 64 + 11) * 2.0 ** -23 * mag + (2.0 ** -25 if t == torch.float16 else 0.0)


# a split-K form with an odd width, one with K inside a panel, the 128 x 128 tiles, the 256 x 256 ones
@pytest.mark.parametrize("rows,n,k", [(90, 51, 320), (700, 96, 1056), (1500, 640, 512), (4096, 4096, 288)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("t", [torch.float16, torch.bfloat16])
def test_calibrated_layer(orc, rows, n, k, with_bias, t):
    g = torch.Generator(device=DEV).manual_seed(rows + n)
    x = torch.randn(rows, k, generator=g, device=DEV) * torch.exp(torch.randn(1, k, generator=g, device=DEV)) + 0.2
    w = torch.randn(n, k, generator=g, device=DEV) * k ** -0.5
    bias = torch.randn(n, generator=g, device=DEV) if with_bias else None
    b64 = 0.0 if bias is None else bias.double()
    y_full = (x.double() @ w.double().t() + b64).float()
    xc, xs, xv = _mx4(x)
    wc, ws, wv = _mx4(w)
    acc, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    # the calibration forward
    y_quant = torch.empty(rows, n, device=DEV)
    P.qlinear_mx4_cwac_forward(xc, xs, wc, ws, None, bias, y_quant)
    y, m = acc + b64, mag + (0.0 if bias is None else b64.abs())
    assert ((y_quant.double() - y).abs() <= _bound(k, y, m, torch.float32)).all()
    # statistics in two batches, the fit
    st = torch.empty(P.cwac_stats_bytes(n) // 8 + 2, dtype=torch.float64, device=DEV)
    part = torch.empty(P.cwac_calibrate_stats_workspace(rows, n), dtype=torch.uint8, device=DEV)
    half = rows // 2 + 1
    P.cwac_calibrate_stats(y_full[:half], y_quant[:half], st, part, first=True)
    P.cwac_calibrate_stats(y_full[half:], y_quant[half:], st, part)
    alpha, beta, mult, fbias = (torch.empty(n, device=DEV) for _ in range(4))
    P.cwac_solve(st, n, alpha, beta)
    a0, b0 = orc.fit(y_full.cpu().numpy(), y_quant.cpu().numpy())
    spread = y_full.double().std(0).cpu().numpy()
    a, b = alpha.cpu().numpy(), beta.cpu().numpy()
    assert np.max(np.abs(a - a0) / np.maximum(np.abs(a0), 1.0)) <= 1e-5
    assert np.max(np.abs(b - b0) / np.maximum(np.abs(b0), spread)) <= 1e-5
    # the fold: evaluated in 64 bits, rounded once
    P.cwac_fold_weight_only(alpha, beta, bias, mult, fbias)
    assert torch.equal(mult, alpha) and torch.equal(fbias, (alpha.double() * b64 + beta.double()).float())
    # the compensated forward
    out = torch.empty(rows, n, dtype=t, device=DEV)
    P.qlinear_mx4_cwac_forward(xc, xs, wc, ws, mult, fbias, out)
    y = acc * mult.double() + fbias.double()
    m = mag * mult.double().abs() + fbias.double().abs()
    assert ((out.double() - y).abs() <= _bound(k, y, m, t)).all()
    # (least squares: no farther from the full-precision outputs, in every channel, than without the compensation; 1e-4 of it for the fit's roundings)
    before, after = ((acc + b64 - y_full) ** 2).sum(0), ((y - y_full) ** 2).sum(0)
    assert (after <= before * (1 + 1e-4)).all()
