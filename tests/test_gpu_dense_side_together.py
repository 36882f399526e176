"""The dense side as a training loop uses it: two normalized linear layers in bf16, their gradients by
the library's backward passes, one clip factor over all of them, and AdamW on the lot; eager and
captured.  The products are torch's; everything between them is compared with the same loop whose
normalization, clipping and optimizer are plain formulas in 64 bits."""
import pytest
import torch

import dense_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16
EPS = 1e-5


class Net:
    """y = LN(x W1) W2 with a norm of its own behind; loss sum(w * LN(.)) for a fixed w."""

    def __init__(self, bits, rows=600, d0=24, d1=200, d2=40):
        gen = torch.Generator().manual_seed(1)

        def draw(*s, scale=1.0):
            return (torch.randn(*s, generator=gen) * scale).to(DEV)

        self.x = draw(rows, d0).to(BF16)
        self.w = draw(rows, d2).to(BF16)
        self.params = [draw(d0, d1, scale=0.2).to(BF16), torch.ones(d1, device=DEV),
                       torch.zeros(d1, device=DEV), draw(d1, d2, scale=0.1).to(BF16),
                       torch.ones(d2, device=DEV), torch.zeros(d2, device=DEV)]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.n_valid = torch.tensor([rows - 7], dtype=torch.int32, device=DEV)
        self.buf = {k: torch.zeros(rows, d, dtype=BF16, device=DEV)
                    for k, d in (("a", d1), ("h", d1), ("b", d2), ("y", d2), ("db", d2), ("da", d1))}
        self.stat = [torch.zeros(rows, device=DEV) for _ in range(4)]
        from paper_2404_04270_amd import AdamW, binding as B
        self.ws = torch.empty(max(B.ss_layernorm_rows_workspace_bytes(rows, d) for d in (d1, d2)),
                              dtype=torch.uint8, device=DEV)
        self.opt = AdamW(self.params, lr=1e-2, weight_decay=0.1, state_bits=bits, master=True,
                         no_decay=[p.dim() == 1 for p in self.params], max_norm=2.0)
        self.opt.set_grads(self.grads)

    def gradients(self):
        from paper_2404_04270_amd import binding as B
        W1, g1, b1, W2, g2, b2 = self.params
        f, n = self.buf, self.n_valid
        torch.matmul(self.x, W1, out=f["a"])
        B.ss_layernorm_rows_forward(f["a"], n, g1, b1, EPS, f["h"], self.stat[0], self.stat[1])
        torch.matmul(f["h"], W2, out=f["b"])
        B.ss_layernorm_rows_forward(f["b"], n, g2, b2, EPS, f["y"], self.stat[2], self.stat[3])
        B.ss_layernorm_rows_backward(self.w, f["b"], n, g2, self.stat[2], self.stat[3], f["db"],
                                     self.grads[4], self.grads[5], self.ws)
        torch.matmul(f["h"].t(), f["db"], out=self.grads[3])
        torch.matmul(f["db"], W2.t().contiguous(), out=f["da"])
        B.ss_layernorm_rows_backward(f["da"], f["a"], n, g1, self.stat[0], self.stat[1], f["da"],
                                     self.grads[1], self.grads[2], self.ws)
        torch.matmul(self.x.t(), f["da"], out=self.grads[0])

    def step(self):
        self.gradients()
        self.opt.step()


@pytest.mark.parametrize("bits", [32, 8])
def test_loop_against_formulas(bits):
    net = Net(bits)
    n = int(net.n_valid)
    L, S = net.opt.list, net.opt.state
    for t in (1, 2, 3):
        masters = [L.of(S.master, k).clone() if p.dtype is BF16 else p.clone()
                   for k, p in enumerate(net.params)]
        if bits == 32:
            m0, v0 = S.m.clone(), S.v.clone()
        else:
            m0 = ref.decode(S.m.cpu(), S.exps[:, 0].cpu(), 14, True).to(DEV)
            v0 = ref.decode(S.v.cpu(), S.exps[:, 1].cpu(), 30, False).to(DEV)
        g1 = net.params[1].clone()
        net.step()
        # the norms inside: y of the first, dgamma and dbeta of the first, as of its own inputs
        a = net.buf["a"][:n]
        y, _, _ = ref.layernorm(a, g1, masters[2], EPS)
        off = (net.buf["h"][:n].double() - y).abs()
        assert not bool((off > ref.half_step(BF16) * y.abs() + 2e-5).any())
        assert not bool(net.buf["h"][n:].any())          # rows that do not count: as they were made
        # clip and step, from the gradients as they are
        norm = torch.stack([g.double().square().sum() for g in net.grads]).sum().sqrt().item()
        assert abs(net.opt.clip[0].item() - norm) <= 2 * ref.HALF32 * norm
        factor = min(1.0, 2.0 / (norm + 1e-6))
        assert abs(net.opt.clip[1].item() - factor) <= 2 * ref.HALF32 * factor
        for k, p in enumerate(net.params):
            want, _, _, tol, _, _ = ref.adamw(masters[k].reshape(-1), net.grads[k].reshape(-1),
                                              L.of(m0, k), L.of(v0, k), t, lr=1e-2,
                                              weight_decay=0.1 if p.dim() == 2 else 0.0,
                                              factor=net.opt.clip[1].item())
            got = L.of(S.master, k) if p.dtype is BF16 else p.reshape(-1)
            assert not bool(((got.double() - want).abs() > tol).any()), (t, k)
            if p.dtype is BF16:
                assert torch.equal(p.reshape(-1), got.to(BF16))
    assert net.opt.steps() == 3


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_loop_replays_like_the_eager_one(bits):
    eager, cap = Net(bits), Net(bits)
    for net in (eager, cap):
        net.step()                                       # libraries set themselves up outside of it
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap.step()
    for k in range(4):
        eager.x.mul_(1.0 - 0.125 * k)
        cap.x.mul_(1.0 - 0.125 * k)
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.params + eager.grads, cap.params + cap.grads):
            assert torch.equal(a, b), k
        assert torch.equal(eager.opt.state.m, cap.opt.state.m)
        assert torch.equal(eager.opt.state.v, cap.opt.state.v)
    assert cap.opt.steps() == 5
