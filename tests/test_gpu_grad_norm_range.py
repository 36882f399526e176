"""Gradient norms above the range of fp32: finite in 64 bits, so the step is taken, clipped by them."""
import pytest
import torch

import dense_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n", [2, 300_000])              # norms of one launch and of two
def test_norm_above_the_range_of_fp32(n):
    from paper_2404_04270_amd import AdamW
    gen = torch.Generator().manual_seed(n)
    g0 = 3e38 * (1 - 2.0 * torch.randint(0, 2, (n,), generator=gen))
    p, g = torch.zeros(n, device=DEV), g0.to(DEV)
    opt = AdamW([p], lr=1e-2, weight_decay=0.0, max_norm=1.0)
    opt.set_grads([g])
    opt.step()
    norm = float(g0.double().square().sum().sqrt())
    assert norm > torch.finfo(torch.float32).max
    assert opt.clip[0].item() == float("inf") and opt.clip[2].item() == 1.0
    assert opt.steps() == 1 and opt.left_out() == 0
    # the factor is subnormal: off by half of 2^-149, and so is what it is multiplied by
    factor = 1.0 / norm
    assert abs(opt.clip[1].item() - factor) <= 2.0 ** -150
    m = opt.list.of(opt.state.m, 0).cpu().double()
    want = 0.1 * factor * g0.double()
    assert not bool(((m - want).abs() > 0.1 * 2.0 ** -150 * g0.double().abs()
                     + 4 * ref.HALF32 * want.abs()).any())
    assert bool(torch.isfinite(p).all())
