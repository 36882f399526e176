"""LayerNorm of rows of 8193 to 16384 columns against 64 bits, with the bound that their splits over
lanes ask for (tests/test_gpu_layernorm_rows.py allows these widths sixteen times as much).

A row belongs to 512 lanes with 32 elements each: a sum is 31 additions in a lane, 6 in the wavefront's
tree and 7 over the wavefronts, so it is off by at most 44 u times the sum of its terms' sizes
(u = 2^-24); with the product by 1 / dim, itself rounded, 46 u.
  mean   46 u size, size = mean |x|; taken as 50
  rstd   the variance's terms are off by 3 u (difference and square), their sum by 44, the product by 2,
         eps's addition by 1: 50 u, of which the root leaves half; root and quotient add 3: 28 u, and
         the mean's error d adds (d rstd)^2 / 2.  Taken as 30 u and that
  y      x - mu is off by u |x - mu| + 50 u size, rstd by 30 u, two roundings more: 34 u |x - mu| rstd +
         51 u size rstd, each times gamma; the sum with beta by a half step
  dx     rstd (g - m1 - xh m2), g = gamma dy off by u, m1 by 47 u of mean |g|, m2 by 48 u of mean |g xh|
         and by what xh is off in it; three roundings and rstd's 30 u in all of it"""
import pytest
import torch

import dense_reference as ref
from test_gpu_layernorm_rows import BF16, DEV, EPS, F16, F32, close, matrix, rounded

pytestmark = pytest.mark.gpu
U = ref.HALF32


@pytest.mark.parametrize("rows,dim", [(1, 8193), (5, 8200), (300, 9001), (515, 11_003), (700, 12_288),
                                      (4, 16_377), (530, 16_384)])
@pytest.mark.parametrize("dtype,wt", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16), (F16, F32)])
def test_rows_of_8_to_16_thousand_columns(rows, dim, dtype, wt):
    from paper_2404_04270_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(rows + dim)
    _, x = matrix(rows, dim, dtype, gen, dim % 3)
    _, dy = matrix(rows, dim, dtype, gen, dim % 3, shift=0.1, scale=0.5)
    gamma = (torch.randn(dim, device=DEV, generator=gen) * 0.2 + 1).to(wt)
    beta = (torch.randn(dim, device=DEV, generator=gen) * 0.2).to(wt)
    y, dx = torch.empty(2, rows, dim, dtype=dtype, device=DEV).unbind(0)
    mean, rstd = torch.empty(2, rows, device=DEV).unbind(0)
    dgamma, dbeta = torch.empty(2, dim, dtype=wt, device=DEV).unbind(0)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
    B.ss_layernorm_rows_forward(x, None, gamma, beta, EPS, y, mean, rstd)
    B.ss_layernorm_rows_backward(dy, x, None, gamma, mean, rstd, dx, dgamma, dbeta, ws)

    want, mu, rs = ref.layernorm(x, gamma, beta, EPS)
    size = x.double().abs().mean(1)
    close(mean, mu, 50 * U * size, "mean")
    away = 30 * U + (50 * U * size * rs) ** 2
    close(rstd, rs, away * rs, "rstd")
    r, ga = rs[:, None], gamma.double().abs()
    c = (x.double() - mu[:, None]).abs()
    off_xh = r * U * (34 * c + 51 * size[:, None])
    close(y, want, rounded(want, off_xh * ga + U * want.abs(), dtype), "y")

    dxw, dgw, dbw, xh, _ = ref.layernorm_backward(dy, x, gamma, EPS)
    g = dy.double().abs() * ga
    m1, m2 = g.mean(1, keepdim=True), (g * xh.abs()).mean(1, keepdim=True)
    off = r * (U * (g + 47 * m1) + xh.abs() * (48 * U * m2 + (g * off_xh).mean(1, keepdim=True))
               + off_xh * m2 + 3 * U * (g + m1 + xh.abs() * m2)) + 30 * U * dxw.abs()
    close(dx, dxw, rounded(dxw, off, dtype), "dx")
    # column sums: at most `rows` terms one after the other or in parts
    t = (dy.double() * xh).abs()
    off = U * (rows + 1) * t.sum(0) + (dy.double().abs() * off_xh).sum(0)
    close(dgamma, dgw, rounded(dgw, off, wt), "dgamma")
    close(dbeta, dbw, rounded(dbw, U * rows * dy.double().abs().sum(0), wt), "dbeta")
