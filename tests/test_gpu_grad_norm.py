"""Norm of many gradients and the clip factor against 64-bit sums.  The kernel's sums are in fp64;
what is off is one rounding to fp32 of each result: half a step."""
import math

import pytest
import torch

import dense_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def norm_of(grads, max_norm, scale=1.0):
    from paper_2404_04270_amd import binding as B
    tl = B.TensorList(grads)
    clip = torch.full((4,), -1.0, device=DEV)
    ws = torch.empty(B.ss_grad_norm_workspace_bytes(tl), dtype=torch.uint8, device=DEV)
    B.ss_grad_norm(tl, max_norm, clip, ws, scale)
    return clip.tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", [[1], [7, 0, 1], [8192], [8193, 1, 16384, 3], [2_000_003],
                                   [65] * 700, [50_000] * 500,
                                   [2048] * 64, [2048] * 65, [131_072], [131_073]])
def test_norm_and_factor(dtype, sizes):
    gen = torch.Generator(device=DEV).manual_seed(len(sizes) + sizes[0])
    flat = torch.randn(sum(sizes) + 1, device=DEV, generator=gen).to(dtype)[1:]
    grads = list(flat.split(sizes))
    want = flat.double().norm().item()
    for max_norm, scale in [(1.0, 1.0), (1e9, 1.0), (0.25, -0.5), (math.inf, 2.0 ** -10)]:
        norm, factor, finite, rest = norm_of(grads, max_norm, scale)
        n = abs(scale) * want
        f = scale * min(1.0, max_norm / (n + 1e-6))
        assert abs(norm - n) <= 2 * ref.HALF32 * n
        assert abs(factor - f) <= 2 * ref.HALF32 * abs(f)
        assert finite == 1.0 and rest == 0.0


def test_several_types_in_one_norm():
    gen = torch.Generator().manual_seed(1)
    grads = [torch.randn(n, generator=gen).to(d).to(DEV) for n, d in
             [(999, torch.float32), (5000, torch.bfloat16), (31, torch.float16), (12345, torch.bfloat16)]]
    want = math.sqrt(sum(g.double().square().sum().item() for g in grads))
    assert abs(norm_of(grads, 1.0)[0] - want) <= 2 * ref.HALF32 * want


def test_values_whose_squares_leave_fp32():
    """1e25 squared is no fp32 number, 1e-25 squared neither: the sums hold both."""
    for x in (1e25, 1e-25):
        g = torch.full((1000,), x, device=DEV)
        want = g.double().norm().item()
        norm, factor, finite, _ = norm_of([g], 1.0)
        assert abs(norm - want) <= 2 * ref.HALF32 * want and finite == 1.0
        assert factor == pytest.approx(min(1.0, 1.0 / (want + 1e-6)), rel=2 * ref.HALF32)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_what_is_not_finite_is_told(bad, dtype):
    g = torch.ones(30_000, dtype=dtype, device=DEV)
    assert norm_of([g[:100], g], 1.0)[2] == 1.0
    for at in (0, 8191, 29_999):
        h = g.clone()
        h[at] = bad
        norm, factor, finite, _ = norm_of([g[:100], h], 1.0)
        assert not math.isfinite(norm) and factor == 0.0 and finite == 0.0


def test_zero_gradients():
    norm, factor, finite, _ = norm_of([torch.zeros(5000, device=DEV)], 1.0)
    assert (norm, factor, finite) == (0.0, 1.0, 1.0)
