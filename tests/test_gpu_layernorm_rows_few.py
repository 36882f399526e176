"""LayerNorm of few rows backward: how many launches a call has on both sides of the border of the one
workgroup that takes all rows, and that both give the definition's gradients."""
import pytest
import torch

import dense_reference as ref
from test_gpu_layernorm_rows import BF16, DEV, EPS, F16, F32, both_ways

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,dim,dtype,launches", [
    (4, 8192, F32, 1), (2, 16_384, BF16, 1), (3, 10_922, F16, 1), (128, 64, F32, 1), (1, 16_384, F32, 1),
    (3, 10_923, F16, 2), (3, 16_384, F32, 2), (4, 16_384, BF16, 2), (4, 9001, BF16, 2),
    (5, 8192, F32, 2), (129, 64, F32, 2), (3, 16_385, F32, 3), (1, 20_000, BF16, 3)])
def test_launches_of_few_rows(rows, dim, dtype, launches):
    from paper_2404_04270_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(dim)
    x, dy = torch.randn(2, rows, dim, device=DEV, generator=gen).to(dtype).unbind(0)
    mu = x.double().mean(1)
    mean, rstd = mu.float(), (1 / (x.double().var(1, correction=0) + EPS).sqrt()).float()
    dx, only = torch.empty_like(x), torch.empty_like(x)
    dg, db = torch.empty(2, dim, dtype=dtype, device=DEV).unbind(0)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
    B.ss_profile_enable(True)
    try:
        B.ss_layernorm_rows_backward(dy, x, None, None, mean, rstd, dx, dg, db, ws)
        torch.cuda.synchronize()
        assert sum(n for n, _ in B.ss_profile_report().values()) == launches
        B.ss_layernorm_rows_backward(dy, x, None, None, mean, rstd, only, None, None, None)
        torch.cuda.synchronize()
        assert sum(n for n, _ in B.ss_profile_report().values()) == 1
    finally:
        B.ss_profile_enable(False)
    assert torch.equal(dx, only)
    # the sum of `rows` values in fp32, rounded once more in 16 bits
    want = dy.double().sum(0)
    tol = ref.HALF32 * rows * dy.double().abs().sum(0)
    if dtype is not F32:
        tol = tol + ref.half_step(dtype) * (want.abs() + tol) + (2.0 ** -25 if dtype is F16 else 0.0)
    assert not bool(((db.double() - want).abs() > tol).any())


@pytest.mark.parametrize("rows,dim,dtype,wt,pad,n_valid", [
    (3, 10_922, F16, F16, 1, None), (3, 10_923, BF16, F32, 2, 2), (4, 16_383, F32, F32, 3, None),
    (2, 16_384, F32, F32, 0, 1), (4, 9001, F16, F32, 0, 0)])
def test_few_wide_rows(rows, dim, dtype, wt, pad, n_valid):
    both_ways(rows, dim, dtype, wt, pad, n_valid, seed=rows + dim)
