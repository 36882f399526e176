"""AdamW where a step takes other ways than in small lists: more than one launch, past the caches,
tensors at even and at odd places, elements beyond 2^31."""
import pytest
import torch

import dense_reference as ref
from test_gpu_adamw import close, codes_agree

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def tensors(sizes, dtype, seed, scale, odd):
    """Views of one buffer, one behind the other (at odd places if the sizes are odd)."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    flat = torch.randn(sum(sizes) + odd, device=DEV, generator=gen).mul_(scale).to(dtype)
    return list(flat[odd:].split(sizes))


def reference(p, g, m, v, t, **kw):
    """dense_reference.adamw on the device."""
    return ref.adamw(p, g, m, v, t, **kw)


# 1024 chunks of 2048 elements and fewer go in one launch; from 8 M elements on a step streams
@pytest.mark.parametrize("dtype,grad_dtype,master", [
    (F32, F32, False), (BF16, BF16, True), (BF16, F32, False), (F16, F16, False), (F16, F32, True)])
@pytest.mark.parametrize("sizes,odd", [([600_000, 1, 4097, 2048], 1), ([1024 * 2048], 0),
                                       ([1024 * 2048 + 1], 0), ([33 * 2048], 0),
                                       ([8_400_000, 2048, 77], 0), ([5_000_001, 3_500_000], 1)])
def test_steps_of_larger_lists(sizes, odd, dtype, grad_dtype, master):
    from paper_2404_04270_amd import AdamW
    ps = tensors(sizes, dtype, 1, 0.05, odd)
    gs = tensors(sizes, grad_dtype, 2, 1e-2, odd)
    opt = AdamW(ps, lr=1e-2, weight_decay=0.1, master=master, grad_dtypes=[grad_dtype] * len(ps))
    opt.set_grads(gs)
    for t in (1, 2):
        old = [(opt.list.of(opt.state.master, k) if master else ps[k]).clone()
               for k in range(len(sizes))]
        m0, v0 = opt.state.m.clone(), opt.state.v.clone()
        opt.step()
        for k in range(len(sizes)):
            p, m, v, tp, tm, tv = reference(old[k], gs[k], opt.list.of(m0, k), opt.list.of(v0, k), t,
                                            lr=1e-2, weight_decay=0.1)
            for got, want, tol in ((opt.list.of(opt.state.m, k), m, tm),
                                   (opt.list.of(opt.state.v, k), v, tv)):
                assert not bool(((got.double() - want).abs() > tol).any()), (t, k)
            if master:
                got = opt.list.of(opt.state.master, k)
                assert torch.equal(ps[k], got.to(dtype))
            else:
                got = ps[k]
                if dtype is not F32:
                    tp = tp + ref.half_step(dtype) * (p.abs() + tp) + (
                        2.0 ** -25 if dtype is F16 else 0.0)
            assert not bool(((got.double() - p).abs() > tp).any()), (t, k)
    assert opt.steps() == 2


@pytest.mark.parametrize("bits", [32, 8])
def test_one_launch_and_two_agree(bits):
    """The same tensor alone and at the head of a list that needs more launches: the same bits."""
    from paper_2404_04270_amd import AdamW
    first = tensors([500_001], F32, 3, 0.05, 0)[0]
    grad = tensors([500_001], F32, 4, 1e-2, 0)[0]
    results = []
    for more in (0, 1_700_000, 9_000_000):
        ps = [first.clone()] + tensors([more], F32, 5, 0.05, 0)
        gs = [grad] + tensors([more], F32, 6, 1e-2, 0)
        opt = AdamW(ps, state_bits=bits)
        opt.set_grads(gs)
        for _ in range(3):
            opt.step()
        results.append([ps[0], opt.list.of(opt.state.m, 0).clone(),
                        opt.list.of(opt.state.v, 0).clone()])
        assert opt.steps() == 3
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


def test_large_list_steps_out_of_a_graph_and_is_left_out():
    from paper_2404_04270_amd import AdamW
    ps, gs = tensors([2_200_000, 513], BF16, 7, 0.05, 0), tensors([2_200_000, 513], BF16, 8, 1e-2, 0)
    twin = [p.clone() for p in ps]
    opts = [AdamW(x, state_bits=8, max_norm=0.5) for x in (ps, twin)]
    for o in opts:
        o.set_grads(gs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opts[1].step()
    for k in range(5):
        keep = gs[0][999].clone()
        if k == 2:
            gs[0][999] = float("inf")
        opts[0].step()
        graph.replay()
        torch.cuda.synchronize()
        gs[0][999] = keep
        gs[0].mul_(1.125)
        assert all(torch.equal(a, b) for a, b in zip(ps, twin)), k
        assert torch.equal(opts[0].state.v, opts[1].state.v)
        assert torch.equal(opts[0].state.counters[:2], opts[1].state.counters[:2])
    assert opts[1].steps() == 4 and opts[1].left_out() == 1


def test_elements_beyond_two_to_the_31():
    """One bf16 tensor of 2^31 + 70001 elements with packed moments: places around 2^31 and at its end
    are looked at, the others by what they share with the first 4096 (the gradient repeats)."""
    from paper_2404_04270_amd import AdamW
    n = 2 ** 31 + 70_001
    gen = torch.Generator(device=DEV).manual_seed(9)
    p = torch.zeros(n, dtype=BF16, device=DEV)
    g = torch.empty(n, dtype=BF16, device=DEV)
    base = torch.randn(4096, device=DEV, generator=gen).to(BF16)
    g[:2 ** 31].view(-1, 4096).copy_(base)
    g[2 ** 31:] = torch.randn(70_001, device=DEV, generator=gen).to(BF16)
    opt = AdamW([p], lr=0.25, weight_decay=0.0, state_bits=8, max_norm=1e30)
    opt.set_grads([g])
    opt.step()
    want = base.double().square().sum().item() * 2 ** 19 + g[2 ** 31:].double().square().sum().item()
    assert abs(opt.clip[0].item() ** 2 - want) <= 4 * ref.HALF32 * want
    assert bool((p[:2 ** 31].view(-1, 4096) == p[:4096]).all())
    for lo, hi in ((0, 4096), (2 ** 31 - 2048, 2 ** 31 + 2048), (n - 3000 - n % 128, n)):
        lo -= lo % 128
        gg = g[lo:hi].cpu()
        zero = torch.zeros(hi - lo)
        pw, m, v, tp, _, _ = ref.adamw(zero, gg, zero, zero, 1, lr=0.25, weight_decay=0.0)
        close(p[lo:hi], pw, tp + ref.half_step(BF16) * pw.abs(), lo)
        pad = torch.zeros(ref.padded(hi) - hi, dtype=torch.float64)
        end, blocks = ref.padded(hi), slice(lo // 128, ref.padded(hi) // 128)
        codes_agree(opt.state.m[lo:end], opt.state.exps[blocks, 0], torch.cat([m, pad]), 14, True, 1,
                    0, lo, ("m", lo))
        codes_agree(opt.state.v[lo:end], opt.state.exps[blocks, 1], torch.cat([v, pad]), 30, False, 1,
                    1 << 31, lo, ("v", lo))


def test_lists_refuse_overlapping_parameters_and_gradients_as_parameters():
    from paper_2404_04270_amd import AdamW, binding as B
    flat = torch.zeros(1000, device=DEV)
    for ps in ([flat, flat], [flat[:600], flat[599:]]):
        with pytest.raises(B.SlipstreamError, match="overlap"):
            AdamW(ps)
    AdamW([flat[:600], flat[600:]])
    norm_only = B.TensorList([flat, flat])
    with pytest.raises(B.SlipstreamError, match="gradients"):
        B.AdamWState(norm_only)
    opt = AdamW([flat])
    with pytest.raises(B.SlipstreamError, match="no gradients yet"):
        opt.step()
    for bad in ([flat[:999]], [flat.to(BF16)], [flat, flat], [torch.zeros(1, device=DEV).expand(1000)],
                [torch.zeros(1000)]):
        with pytest.raises(B.SlipstreamError, match="grads"):
            opt.set_grads(bad)
    with pytest.raises(B.SlipstreamError):
        AdamW([torch.zeros(10, 10, device=DEV).t()])
    with pytest.raises(B.SlipstreamError):
        AdamW([flat], grad_dtypes=[BF16])
    with pytest.raises(B.SlipstreamError):
        AdamW([flat], grad_scale=0.5)
    with pytest.raises(B.SlipstreamError, match="another list"):
        B.ss_adamw_step(B.TensorList([flat[:10]], grads=[flat[:10].clone()]), opt.state, 1e-3)
    with pytest.raises(B.SlipstreamError, match="bits"):
        opt.moments(torch.empty(1024, dtype=BF16, device=DEV), torch.empty(1024, dtype=BF16, device=DEV))


@pytest.mark.parametrize("bits", [32, 8])
def test_lists_without_elements(bits):
    from paper_2404_04270_amd import AdamW
    opt = AdamW([torch.zeros(0, device=DEV)], state_bits=bits, max_norm=1.0)
    opt.set_grads([torch.zeros(0, device=DEV)])
    opt.step()
    assert opt.steps() == 1 and opt.clip.tolist() == [0.0, 1.0, 1.0, 0.0]
