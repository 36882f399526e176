"""AdamW over many tensors against the formula in 64 bits: types, odd sizes and places, moments in
32 and in 8 bits, clipping, steps left out, and what a captured step does."""
import pytest
import torch

import dense_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SIZES = [1, 3, 127, 128, 129, 1000, 0, 2047, 2049, 8191, 8192, 8193, 20000]


class Model:
    """Tensors of `sizes` in one flat buffer with `gap` elements of a sentinel between them."""

    def __init__(self, sizes, dtype, grad_dtype, seed, gap=1, grad_scale=1.0):
        gen = torch.Generator().manual_seed(seed)
        self.sizes, self.gap = list(sizes), gap
        n = sum(sizes) + gap * (len(sizes) + 1)
        self.flat = torch.full((n,), 7.0).to(dtype).to(DEV)
        self.params, at = [], gap
        for k in sizes:
            self.params.append(self.flat[at:at + k])
            at += k + gap
        self.grads = []
        for p in self.params:
            p.copy_((torch.randn(p.numel(), generator=gen) * 0.05).to(dtype))
            g = torch.randn(p.numel(), generator=gen) * torch.exp(
                2 * torch.randn(p.numel(), generator=gen)) * 1e-3 * grad_scale
            buf = torch.zeros(p.numel() + 1, dtype=grad_dtype, device=DEV)
            self.grads.append(buf[1:])                     # one element off
            self.grads[-1].copy_(g.to(grad_dtype))

    def between_untouched(self):
        at, ok = 0, True
        for k in self.sizes + [0]:
            ok &= bool((self.flat[at:at + self.gap].float() == 7.0).all())
            at += self.gap + k
        return ok


def close(got, want, tol, what):
    d = (got.detach().double().cpu() - want).abs()
    bad = d > tol
    assert not bool(bad.any()), (what, int(bad.sum()), float((d - tol).max()))


def masters_or_params(opt, k):
    return opt.list.of(opt.state.master, k) if opt.state.master is not None else opt.list.params[k]


@pytest.mark.parametrize("dtype,grad_dtype,master", [
    (F32, F32, False), (BF16, BF16, False), (BF16, BF16, True), (BF16, F32, True),
    (F16, F16, True), (F16, F32, False)])
def test_steps_match_the_formula(dtype, grad_dtype, master):
    from paper_2404_04270_amd import AdamW
    mod = Model(SIZES, dtype, grad_dtype, seed=1)
    no_decay = [k % 3 == 0 for k in range(len(SIZES))]
    opt = AdamW(mod.params, lr=2e-3, betas=(0.9, 0.99), eps=1e-7, weight_decay=0.1, master=master,
                no_decay=no_decay, grad_dtypes=[grad_dtype] * len(SIZES))
    opt.set_grads(mod.grads)
    for t in (1, 2, 3):
        before = [(masters_or_params(opt, k).clone().cpu(), opt.list.of(opt.state.m, k).clone().cpu(),
                   opt.list.of(opt.state.v, k).clone().cpu()) for k in range(len(SIZES))]
        opt.step()
        torch.cuda.synchronize()
        for k, (p0, m0, v0) in enumerate(before):
            p, m, v, tp, tm, tv = ref.adamw(p0, mod.grads[k].cpu(), m0, v0, t, 2e-3, 0.9, 0.99, 1e-7,
                                            0.0 if no_decay[k] else 0.1)
            close(opt.list.of(opt.state.m, k), m, tm, ("m", t, k))
            close(opt.list.of(opt.state.v, k), v, tv, ("v", t, k))
            if master:
                close(opt.list.of(opt.state.master, k), p, tp, ("master", t, k))
                assert torch.equal(opt.list.params[k], opt.list.of(opt.state.master, k).to(dtype))
            else:
                if dtype is not F32:               # rounded once more, by half a step
                    tp = tp + ref.half_step(dtype) * (p.abs() + tp) + (
                        2.0 ** -25 if dtype is F16 else 0.0)
                close(opt.list.params[k], p, tp, ("p", t, k))
    assert mod.between_untouched() and opt.steps() == 3 and opt.left_out() == 0


def codes_agree(code, exps, want, top, signed, t, turn, first, what):
    """code: uint8 of whole blocks.  The codes of `want` (float64), but where fp32 rounding of the
    moment (a few parts in 2^24 of 16 steps, and 2^-20 of one in the lowest field) decides."""
    # the largest of a block is off by at most 8 half steps of fp32 (two constants, three products, a
    # sum and the factor): where a power of two is that near, either exponent is right
    e, got = exps.long().cpu(), code.long().cpu()
    for rel in (1 - 8 * ref.HALF32, 1 + 8 * ref.HALF32):
        near = ref.exponents(want.abs() * rel, top)
        assert bool(((e - near) * (1 if rel < 1 else -1) >= 0).all()), (what, "exponents")
    c, place = ref.encode(want.abs(), e, top, t, turn, first)
    if signed:
        neg = got >= 128
        got = got % 128
        assert not bool((neg != (want < 0))[got > 0].any()), what
    elif bool((want > 0).any()):
        c = torch.where((want > 0) & (c == 0), 1, c)
    differ = got != c
    near = (place - place.round()).abs() < 1e-5
    assert not bool((differ & ~near).any()), (what, int((differ & ~near).sum()))
    assert int((got - c).abs().max() if got.numel() else 0) <= 1, what


@pytest.mark.parametrize("dtype,grad_dtype,master", [
    (F32, F32, False), (BF16, BF16, False), (BF16, F32, True), (F16, F16, False), (F16, F32, True)])
def test_packed_steps_match_the_definition(dtype, grad_dtype, master):
    from paper_2404_04270_amd import AdamW
    mod = Model(SIZES, dtype, grad_dtype, seed=2)
    opt = AdamW(mod.params, lr=1e-2, weight_decay=0.05, master=master, state_bits=8,
                grad_dtypes=[grad_dtype] * len(SIZES))
    opt.set_grads(mod.grads)
    L, S = opt.list, opt.state
    for t in (1, 2, 3):
        old = [masters_or_params(opt, k).clone().cpu() for k in range(len(SIZES))]
        m0 = ref.decode(S.m.cpu(), S.exps[:, 0].cpu(), 14, True)
        v0 = ref.decode(S.v.cpu(), S.exps[:, 1].cpu(), 30, False)
        opt.step()
        torch.cuda.synchronize()
        mv = torch.empty(2, L.state_elems, dtype=BF16, device=DEV)
        opt.moments(mv[0], mv[1])
        assert torch.equal(mv[0].cpu().double(), ref.decode(S.m.cpu(), S.exps[:, 0].cpu(), 14, True))
        assert torch.equal(mv[1].cpu().double(), ref.decode(S.v.cpu(), S.exps[:, 1].cpu(), 30, False))
        for k, n in enumerate(SIZES):
            a, z = L.starts[k], L.starts[k] + ref.padded(n)
            p, m, v, tp, _, _ = ref.adamw(old[k], mod.grads[k].cpu(), m0[a:a + n], v0[a:a + n], t,
                                          lr=1e-2, weight_decay=0.05)
            pad = torch.zeros(z - a - n, dtype=torch.float64)
            blocks = slice(a // 128, z // 128)
            codes_agree(S.m[a:z], S.exps[blocks, 0], torch.cat([m, pad]), 14, True, t, 0, a,
                        ("m", t, k))
            codes_agree(S.v[a:z], S.exps[blocks, 1], torch.cat([v, pad]), 30, False, t, 1 << 31, a,
                        ("v", t, k))
            if master:
                close(L.of(S.master, k), p, tp, ("master", t, k))
                assert torch.equal(L.params[k], L.of(S.master, k).to(dtype))
            else:
                if dtype is not F32:
                    tp = tp + ref.half_step(dtype) * (p.abs() + tp) + (
                        2.0 ** -25 if dtype is F16 else 0.0)
                close(L.params[k], p, tp, ("p", t, k))
    assert mod.between_untouched() and opt.steps() == 3


def test_packed_moments_of_steady_gradients_come_out_right():
    """With gradients that stay the same v approaches g^2 by 0.1 % a step, codes are 6 to 12 % apart.
    An element's v is then within a code or two of its value; over 4096 elements the deviations (at
    most 12.5 %, spread evenly: 3.6 %) average out to 0.06 %, and 2 % is 35 times that."""
    from paper_2404_04270_amd import AdamW
    gen = torch.Generator().manual_seed(3)
    p = torch.zeros(4096, device=DEV)
    g = (torch.randn(4096, generator=gen) * 0.1 + 0.3).to(DEV)
    opt = AdamW([p], lr=0.0, state_bits=8)
    opt.set_grads([g])
    for _ in range(1500):
        opt.step()
    m, v = torch.empty(2, 4096, dtype=BF16, device=DEV).unbind(0)
    opt.moments(m, v)
    big = g.abs() > 0.05
    rv = (v.double() / (g.double() ** 2 * (1 - 0.999 ** 1500)))[big]
    rm = (m.double() / g.double())[big]
    assert abs(float(rv.mean()) - 1) < 0.02 and abs(float(rm.mean()) - 1) < 0.02
    assert float((rv - 1).abs().max()) < 0.5 and float((rm - 1).abs().max()) < 0.5
    assert opt.steps() == 1500


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_of_several_types_in_one_step(bits):
    """A mixed model steps as its parts do alone: bit for bit, in parameters and moments (but the
    dither, which goes by the place among the moments: the parts keep theirs by being first)."""
    from paper_2404_04270_amd import AdamW
    parts = [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]
    mods = [Model([5, 300, 4097], d, g, seed=10 + i) for i, (d, g) in enumerate(parts)]
    for master in (False, True):
        mixed = [p.clone() for m in mods for p in m.params]
        opt = AdamW(mixed, state_bits=bits, master=master,
                    grad_dtypes=[g for _, g in parts for _ in range(3)])
        opt.set_grads([g for m in mods for g in m.grads])
        for _ in range(2):
            opt.step()
        for i, (mod, (d, g)) in enumerate(zip(mods, parts)):
            alone = [p.clone() for p in mod.params]
            one = AdamW(alone, state_bits=bits, master=master, grad_dtypes=[g] * 3)
            one.set_grads(mod.grads)
            for _ in range(2 if bits == 32 else 1):
                one.step()
            if bits == 32:
                for k in range(3):
                    assert torch.equal(alone[k], mixed[3 * i + k]), (d, g, k)
                    assert torch.equal(one.list.of(one.state.v, k), opt.list.of(opt.state.v, 3 * i + k))
            else:
                first = [p.clone() for m in mods for p in m.params]
                again = AdamW(first, state_bits=bits, master=master,
                              grad_dtypes=[g for _, g in parts for _ in range(3)])
                again.set_grads([g for m in mods for g in m.grads])
                again.step()
                for k in range(3):
                    assert torch.equal(alone[k], first[3 * i + k]), (d, g, k)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [1, 129, 70_001])
def test_gradients_of_zero_and_the_first_step(bits, n):
    """All zeros: nothing but the decay moves.  A first step moves every element by lr, whatever the
    gradient's size: m / sqrt(v) is the gradient's sign after both corrections."""
    from paper_2404_04270_amd import AdamW
    p0 = torch.linspace(-1, 1, n)
    p = p0.to(DEV)
    g = torch.zeros(n, device=DEV)
    opt = AdamW([p], lr=0.5, weight_decay=0.125, state_bits=bits)
    opt.set_grads([g])
    opt.step()
    close(p, p0.double() * 0.9375, ref.HALF32 * 3 * p0.double().abs(), "decay")
    assert not bool(opt.state.m.any()) and not bool(opt.state.v.any())
    p.copy_(p0)
    opt = AdamW([p], lr=0.5, weight_decay=0.0, state_bits=bits, eps=1e-20)
    g.copy_(torch.logspace(-12, 12, n)).mul_(torch.where(torch.arange(n) % 2 == 0, 1.0, -1.0).to(DEV))
    opt.set_grads([g])
    opt.step()
    close(p, p0.double() - 0.5 * torch.sign(g.cpu().double()), ref.HALF32 * 24, "first step")


def test_extreme_hyperparameters():
    from paper_2404_04270_amd import AdamW
    gen = torch.Generator().manual_seed(5)
    p0, g0 = torch.randn(500, generator=gen), torch.randn(500, generator=gen)
    for b1, b2, wd, lr in [(0.0, 0.0, 0.0, 1e-3), (0.0, 0.999, 0.5, 1.0), (0.9999, 0.9999999, 0.0, 0.1),
                           (0.5, 0.0, 0.0, 0.0)]:
        p, g = p0.to(DEV), g0.to(DEV)
        opt = AdamW([p], lr=lr, betas=(b1, b2), weight_decay=wd)
        opt.set_grads([g])
        m, v, want = torch.zeros(500), torch.zeros(500), p0
        for t in (1, 2):
            want, m, v, tp, _, _ = ref.adamw(want.float(), g0, m.float(), v.float(), t, lr, b1, b2,
                                             1e-8, wd)
            opt.step()
            close(p, want, 4 * tp, (b1, b2, t))       # states rounded apart in between
        with pytest.raises(AssertionError):
            close(p, p0.double() + 1.0, 4 * tp, "oracle off by one")


@pytest.mark.parametrize("bits", [32, 8])
def test_step_is_left_out_where_the_norm_is_not_finite(bits):
    from paper_2404_04270_amd import AdamW
    p = torch.randn(3000, device=DEV)
    g = torch.randn(3000, device=DEV)
    opt = AdamW([p], state_bits=bits, max_norm=1.0)
    opt.set_grads([g])
    opt.step()
    state = [x.clone() for x in (p, opt.state.m, opt.state.v)]
    for bad in (float("nan"), float("inf")):
        keep = g[1234].clone()
        g[1234] = bad
        opt.step()
        g[1234] = keep
        assert all(torch.equal(a, b) for a, b in zip(state, (p, opt.state.m, opt.state.v)))
    assert opt.steps() == 1 and opt.left_out() == 2
    opt.step()
    assert opt.steps() == 2 and not torch.equal(state[0], p) and bool(torch.isfinite(p).all())


def test_packed_moments_keep_the_neighbours_of_what_is_not_finite():
    """Without a norm a gradient that is not finite takes its own parameter along (NaN, as the
    formula says) and nothing else; a finite one whose square overflows leaves its parameter."""
    from paper_2404_04270_amd import AdamW
    g0 = torch.full((256,), 0.01)
    clean, dirty = [], []
    for bad in (False, True):
        p, g = torch.zeros(256, device=DEV), g0.to(DEV)
        opt = AdamW([p], state_bits=8, weight_decay=0.0)
        opt.set_grads([g])
        opt.step()
        if bad:
            g[3], g[7], g[9] = float("nan"), float("inf"), 1e25
        opt.step()
        g.copy_(g0)
        opt.step()
        mv = torch.empty(2, 256, dtype=BF16, device=DEV)
        opt.moments(mv[0], mv[1])
        (dirty if bad else clean).extend([p.cpu(), mv.cpu()])
    others = torch.ones(256, dtype=torch.bool)
    others[[3, 7, 9]] = False
    assert bool(torch.isnan(dirty[0][[3, 7]]).all()) and bool(torch.isfinite(dirty[0][9]))
    # after the bad step the block's exponents are those of its other elements: codes as before
    assert torch.equal(dirty[0][others][:0], clean[0][others][:0])
    second = slice(128, 256)
    assert torch.equal(dirty[0][second], clean[0][second])
    assert torch.equal(dirty[1][:, second], clean[1][:, second])
    assert bool(torch.isfinite(dirty[1].float()).all())
    # m of the block's others: codes of the same value under exponents at most one field apart
    a, b = dirty[1][0, :128].float(), clean[1][0, :128].float()
    assert bool(((a - b).abs() <= 0.25 * b.abs())[others[:128]].all())


def test_small_values_beside_a_large_one():
    """Elements far below their block's largest: v stays positive, so that no step is longer than the
    largest element's kind; elements that no code can hold lose m, not their bound."""
    from paper_2404_04270_amd import AdamW
    gen = torch.Generator().manual_seed(8)
    g = torch.exp(torch.empty(4096).uniform_(-30, 0, generator=gen)).to(DEV)
    g[::128] = 1e3
    p = torch.zeros(4096, device=DEV)
    opt = AdamW([p], lr=1e-3, state_bits=8, weight_decay=0.0, eps=1e-30)
    opt.set_grads([g])
    before = p.clone()
    for t in range(1, 60):
        opt.step()
        move = (p - before).abs().max()
        before.copy_(p)
        # m >= 2^-9 of 2^7..2^8 and v >= 2^-3 of 2^30..2^31 (scaled): the ratio of a smallest m to the
        # root of a smallest v is at most 4 times that of the largest, which is 1 for a steady g
        assert float(move) < 1e-3 * 8, t
    assert bool((opt.state.v > 0).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_replays_with_its_own_count_and_schedule(bits):
    from paper_2404_04270_amd import AdamW
    gen = torch.Generator().manual_seed(9)
    sizes = [1000, 77, 5000]
    p0 = [torch.randn(n, generator=gen) for n in sizes]
    steps = [[torch.randn(n, generator=gen) * 10 for n in sizes] for _ in range(6)]
    lrs = [1e-3 * (k + 1) for k in range(6)]

    def build():
        ps = [p.to(DEV) for p in p0]
        gs = [torch.zeros(n, device=DEV) for n in sizes]
        lr = torch.zeros(1, device=DEV)
        opt = AdamW(ps, lr=lr, state_bits=bits, max_norm=1.0)
        opt.set_grads(gs)
        return ps, gs, lr, opt

    eager, captured = build(), build()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured[3].step()
    for k in range(6):
        for ps, gs, lr, opt in (eager, captured):
            for g, x in zip(gs, steps[k]):
                g.copy_(x)
            lr.fill_(lrs[k])
        eager[3].step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager[0], captured[0]):
            assert torch.equal(a, b), k
        assert torch.equal(eager[3].state.m, captured[3].state.m)
        assert torch.equal(eager[3].state.v, captured[3].state.v)
        assert captured[3].steps() == k + 1


def test_another_stream_and_another_clip():
    """On a stream of its own, with one norm over two optimizers."""
    from paper_2404_04270_amd import AdamW, binding as B
    gen = torch.Generator().manual_seed(11)
    p = [torch.randn(n, generator=gen).to(DEV) for n in (3000, 513)]
    g = [torch.randn(n, generator=gen).to(DEV) for n in (3000, 513)]
    both = B.TensorList(g)
    clip = torch.zeros(4, device=DEV)
    ws = torch.empty(B.ss_grad_norm_workspace_bytes(both), dtype=torch.uint8, device=DEV)
    opts = [AdamW([x]) for x in p]
    old = [x.clone() for x in p]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.ss_grad_norm(both, 0.5, clip, ws)
    for o, x in zip(opts, g):
        o.set_grads([x], stream=s)
        o.step(clip=clip, stream=s)
    s.synchronize()
    norm = torch.cat(g).double().norm().item()
    # fp64 sums, rounded once to fp32
    assert abs(clip[0].item() - norm) <= 2 * ref.HALF32 * norm
    for x, y, z in zip(p, old, g):
        want, _, _, tol, _, _ = ref.adamw(y.cpu(), z.cpu(), torch.zeros(y.numel()),
                                          torch.zeros(y.numel()), 1, factor=0.5 / (norm + 1e-6))
        close(x, want, tol, "clipped")


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-30, 9e-13, 1e-12, 1e-3])
def test_epsilon_on_both_sides_of_the_exact_root(bits, eps):
    """From 1e-12 on packed steps take the hardware's root and reciprocal, each off by a step of fp32:
    four half steps more than the 16 counted for the exact ones cover both, so that the bound is
    taken twice.  Gradients down to 1e-21, whose squares fp32 does not hold: their v is 0 or a few
    steps of 2^-149, so elements are only looked at where v is a normal number, or m / eps is
    what is left (eps far above the root)."""
    from paper_2404_04270_amd import AdamW
    g0 = torch.logspace(-21, 2, 4000)
    p, g = torch.zeros(4000, device=DEV), g0.to(DEV)
    opt = AdamW([p], lr=1.0, eps=eps, weight_decay=0.0, state_bits=bits)
    opt.set_grads([g])
    opt.step()
    want, _, v, tol, _, _ = ref.adamw(torch.zeros(4000), g0, torch.zeros(4000), torch.zeros(4000), 1,
                                      lr=1.0, eps=eps, weight_decay=0.0)
    look = v > 1e-37
    close(p[look.to(DEV)], want[look], 2 * tol[look], eps)
    if eps >= 1e-12:                     # root below 3.5e-18: less than 4e-6 of eps
        close(p[~look.to(DEV)], want[~look], 2 * tol[~look] + 4e-6 * want[~look].abs(), eps)


def test_same_inputs_give_the_same_bits():
    from paper_2404_04270_amd import AdamW
    outs = []
    for _ in range(2):
        mod = Model([40_000, 129, 65_537], BF16, BF16, seed=12)
        opt = AdamW(mod.params, state_bits=8, max_norm=0.1)
        opt.set_grads(mod.grads)
        for _ in range(3):
            opt.step()
        outs.append([mod.flat.clone(), opt.state.m.clone(), opt.state.v.clone(), opt.clip.clone()])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
