"""Layer norm of matrix rows against 64 bits: every split of a row over lanes, both sides of each
border, odd widths, strides and places, types, rows that do not count.

Tolerances.  With u = 2^-24, r = rstd and a = the row's largest |x - mu|: a sum of dim terms in
fp32, taken lane by lane and then over lanes, is off by less than 40 u times the sum of its terms'
sizes (at most 32 terms per lane, 10 steps of the lanes' tree; 16 times as many where a wide row's
lanes loop), counted once for the mean and once for the variance.  y is then off by
u * (100 (|x-mu| + |mu|_1) r + 4 |beta| + ...), taken below with the mean of |x| for |mu|_1.
Results in 16 bits are rounded once more, by half a step."""
import pytest
import torch

import dense_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-5
U = ref.HALF32

# both sides of every border: lanes of 4 (fp32) or 8 elements, 1 to 64 of them, 2 and 4 vectors per
# lane, 256 and 1024 lanes, and what a workgroup's registers do not hold
DIMS = [1, 2, 3, 4, 5, 7, 8, 9, 13, 16, 17, 31, 33, 64, 65, 100, 128, 129, 255, 256, 257, 511, 513,
        1001, 1024, 1025, 2048, 2049, 4095, 4097, 8192, 8193, 16384, 16385, 32768, 32769]


def matrix(rows, dim, dtype, gen, pad, shift=0.5, scale=1.0):
    """[rows, dim] cut out of a wider buffer that starts one element off, sentinels around it."""
    buf = torch.full((rows * (dim + pad) + 1,), 7.0, device=DEV).to(dtype)
    x = buf[1:].view(rows, dim + pad)[:, :dim]
    x.copy_((torch.randn(rows, dim, device=DEV, generator=gen) * scale + shift).to(dtype))
    return buf, x


def rounded(want, tol, dtype):
    if dtype is F32:
        return tol
    return tol + ref.half_step(dtype) * (want.abs() + tol) + (2.0 ** -25 if dtype is F16 else 0.0)


def close(got, want, tol, what):
    d = (got.double() - want).abs()
    bad = d > tol
    assert not bool(bad.any()), (what, int(bad.sum()), float((d - tol).max()))


def untouched(buf, x, rows, dim, pad, n):
    wide = buf[1:].view(rows, dim + pad)
    return (float(buf[0]) == 7.0 and bool((wide[:, dim:].float() == 7.0).all())
            and bool((wide[n:].float() == 7.0).all()))


def both_ways(rows, dim, dtype, wt, pad, n_valid, seed):
    from paper_2404_04270_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = rows if n_valid is None else n_valid
    nv = None if n_valid is None else torch.tensor([n_valid], dtype=torch.int32, device=DEV)
    _, x = matrix(rows, dim, dtype, gen, pad)
    _, dy = matrix(rows, dim, dtype, gen, pad, shift=0.1, scale=0.5)
    gamma = (torch.randn(dim, device=DEV, generator=gen) * 0.2 + 1).to(wt)
    beta = (torch.randn(dim, device=DEV, generator=gen) * 0.2).to(wt)
    ybuf, y = matrix(rows, dim, dtype, gen, pad)
    ybuf.fill_(7.0)
    dbuf, dx = matrix(rows, dim, dtype, gen, pad)
    dbuf.fill_(7.0)
    mean, rstd = torch.full((2, rows), 7.0, device=DEV).unbind(0)
    dgamma, dbeta = torch.full((2, dim), 7.0, device=DEV).to(wt).unbind(0)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
    B.ss_layernorm_rows_forward(x, nv, gamma, beta, EPS, y, mean, rstd)
    B.ss_layernorm_rows_backward(dy, x, nv, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    torch.cuda.synchronize()
    assert untouched(ybuf, y, rows, dim, pad, n) and untouched(dbuf, dx, rows, dim, pad, n)
    assert bool((mean[n:] == 7.0).all()) and bool((rstd[n:] == 7.0).all())

    x, dy, y, dx = x[:n], dy[:n], y[:n], dx[:n]
    k = 16 if dim > 8192 else 1                    # lanes that loop over a wide row
    want, mu, rs = ref.layernorm(x, gamma, beta, EPS)
    size = x.double().abs().mean(1)
    close(mean[:n], mu, k * 50 * U * (size + 1e-30), "mean")
    # var is off by 40 u of itself and by what the mean's error adds; rstd by half of that and the
    # root and the quotient
    away = k * 60 * U * (1 + size * size * rs * rs * 50 * U)
    close(rstd[:n], rs, away * rs, "rstd")
    c = (x.double() - mu[:, None]).abs()
    off = k * U * 100 * rs[:, None] * (c + size[:, None]) * gamma.double().abs() \
        + 4 * U * (beta.double().abs() + want.abs())
    close(y, want, rounded(want, off, dtype), "y")

    dxw, dgw, dbw, xh, _ = ref.layernorm_backward(dy, x, gamma, EPS)
    g = (dy.double() * gamma.double()).abs()
    off_xh = k * U * 100 * rs[:, None] * (c + size[:, None])          # of x-hat, as of y
    m1, m2 = g.mean(1, keepdim=True), (g * xh.abs()).mean(1, keepdim=True)
    off = rs[:, None] * (k * 60 * U * (g + m1 + xh.abs() * m2) + off_xh * m2
                         + xh.abs() * (g * off_xh).mean(1, keepdim=True)) + k * 60 * U * dxw.abs()
    close(dx, dxw, rounded(dxw, off, dtype), "dx")
    # column sums: up to n terms, one workgroup's in turn, then the workgroups'; 1.5 sqrt(n) + 20
    # half steps of the terms' sizes cover both (roundings of either sign), and x-hat's own error
    t = (dy.double() * xh).abs()
    grow = 1.5 * max(n, 1) ** 0.5 + 20
    off = U * grow * t.sum(0) + (dy.double().abs() * off_xh).sum(0)
    close(dgamma, dgw, rounded(dgw, off, wt), "dgamma")
    close(dbeta, dbw, rounded(dbw, U * grow * dy.double().abs().sum(0), wt), "dbeta")


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("dtype,wt", [(F32, F32), (BF16, F32), (F16, F16)])
def test_every_split_of_a_row(dim, dtype, wt):
    rows = 37 if dim <= 2049 else 5
    both_ways(rows, dim, dtype, wt, pad=dim % 4, n_valid=None, seed=dim)


@pytest.mark.parametrize("rows,dim,dtype,wt,pad,n_valid", [
    (1, 1, BF16, BF16, 0, None), (1, 4096, BF16, BF16, 0, None), (3, 100_000, F32, F32, 3, None),
    (3, 100_000, BF16, BF16, 0, 2), (7, 64, F32, F32, 0, 0), (2, 20_000, F16, F32, 0, 0),
    (300, 40, F16, F32, 24, 299), (5000, 13, F32, F32, 0, 4999), (70_001, 8, BF16, F32, 0, None),
    # one workgroup takes all rows (4 per group of lanes) and just not; results past the caches from 32 MB
    # on, inputs from 256 MB on
    (128, 64, F32, F32, 0, None), (129, 64, F32, F32, 0, None), (32, 1000, BF16, BF16, 1, 31),
    (33, 1000, BF16, F32, 0, None), (4, 8192, F16, F16, 0, 3), (3, 16384, BF16, F32, 0, None),
    (16400, 1024, BF16, BF16, 0, 16399), (16400, 1023, F32, F32, 1, None),
    (22000, 2048, F32, F32, 0, None), (45001, 2047, F16, F16, 0, 45000),
    (2500, 512, BF16, BF16, 5, 2047), (3001, 1024, F32, F32, 0, None), (1500, 6000, F16, F16, 1, 1499)])
def test_rows_strides_and_valid_counts(rows, dim, dtype, wt, pad, n_valid):
    both_ways(rows, dim, dtype, wt, pad, n_valid, seed=rows + dim)


@pytest.mark.parametrize("rows,dim,dtype,wt,pad,n_valid", [
    (700, 9001, F16, F16, 1, 699), (530, 12_001, BF16, F32, 0, None), (515, 16_384, F32, F32, 0, 514),
    (770, 16_383, BF16, BF16, 3, None), (258, 8193, F32, F32, 2, None),
    (5000, 12_000, BF16, BF16, 0, None)])
def test_workgroups_with_several_wide_rows(rows, dim, dtype, wt, pad, n_valid):
    both_ways(rows, dim, dtype, wt, pad, n_valid, seed=rows + dim)


@pytest.mark.parametrize("dim", [5, 300, 3000, 50_000])
def test_in_place_and_without_parameters(dim):
    from paper_2404_04270_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(dim)
    x = torch.randn(9, dim, device=DEV, generator=gen)
    dy = torch.randn(9, dim, device=DEV, generator=gen)
    mean, rstd = torch.empty(2, 9, device=DEV).unbind(0)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(9, dim), dtype=torch.uint8, device=DEV)
    y, one, zero = torch.empty_like(x), torch.ones(dim, device=DEV), torch.zeros(dim, device=DEV)
    B.ss_layernorm_rows_forward(x, None, one, zero, EPS, y, mean, rstd)
    z = x.clone()
    B.ss_layernorm_rows_forward(z, None, None, None, EPS, z, mean, rstd)
    assert torch.equal(y, z)
    dx, dg, db = torch.empty_like(x), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    B.ss_layernorm_rows_backward(dy, x, None, one, mean, rstd, dx, dg, db, ws)
    for over in ("dy", "x"):
        a, b = dy.clone(), x.clone()
        dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
        out = a if over == "dy" else b
        B.ss_layernorm_rows_backward(a, b, None, None, mean, rstd, out, dg2, db2, ws)
        assert torch.equal(out, dx) and torch.equal(dg, dg2) and torch.equal(db, db2)
    only = torch.empty_like(dg)
    B.ss_layernorm_rows_backward(dy, x, None, None, mean, rstd, torch.empty_like(x), None, only, ws)
    assert torch.equal(only, db)
    alone = torch.empty_like(x)
    B.ss_layernorm_rows_backward(dy, x, None, None, mean, rstd, alone, None, None, None)
    assert torch.equal(alone, dx)


def test_no_rows_at_all():
    from paper_2404_04270_amd import binding as B
    x = torch.empty(0, 24, device=DEV)
    dg, db = torch.full((2, 24), 7.0, device=DEV).unbind(0)
    none = torch.empty(0, device=DEV)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(0, 24), dtype=torch.uint8, device=DEV)
    B.ss_layernorm_rows_forward(x, None, None, None, EPS, x, none, none)
    B.ss_layernorm_rows_backward(x, x, None, None, none, none, x, dg, db, ws)
    assert not bool(dg.any()) and not bool(db.any())


@pytest.mark.parametrize("dim", [40, 700, 9000])
def test_gradient_against_differences(dim):
    """Central differences of sum(dy * y) in 64 bits along a few directions: with a step of 1e-4 the
    quotient is off by about 1e-8 of the third derivative, far below the kernel's own 1e-5."""
    from paper_2404_04270_amd import binding as B
    gen = torch.Generator().manual_seed(dim)
    x, dy = torch.randn(4, dim, generator=gen), torch.randn(4, dim, generator=gen)
    gamma, beta = torch.randn(dim, generator=gen), torch.randn(dim, generator=gen)
    d = [t.to(DEV) for t in (x, dy, gamma)]
    mean, rstd = torch.empty(2, 4, device=DEV).unbind(0)
    dx, dg, db = torch.empty(4, dim, device=DEV), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(4, dim), dtype=torch.uint8, device=DEV)
    y = torch.empty(4, dim, device=DEV)
    B.ss_layernorm_rows_forward(d[0], None, d[2], beta.to(DEV), EPS, y, mean, rstd)
    B.ss_layernorm_rows_backward(d[1], d[0], None, d[2], mean, rstd, dx, dg, db, ws)

    def value(a, b, c):
        return float((dy.double() * ref.layernorm(a, b, c, EPS)[0]).sum())

    h = 1e-4
    for _ in range(3):
        ex, eg, eb = (torch.randn(s, generator=gen).double() for s in ((4, dim), (dim,), (dim,)))
        num = (value(x + h * ex, gamma + h * eg, beta + h * eb)
               - value(x - h * ex, gamma - h * eg, beta - h * eb)) / (2 * h)
        parts = [(dx.cpu().double() * ex), (dg.cpu().double() * eg), (db.cpu().double() * eb)]
        got = sum(float(p.sum()) for p in parts)
        size = sum(float(p.abs().sum()) for p in parts)
        assert abs(got - num) <= 1e-5 * size


def test_captured_passes_replay():
    from paper_2404_04270_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(4)
    x, dy = torch.randn(2, 700, 320, device=DEV, generator=gen).to(BF16).unbind(0)
    gamma, beta = torch.randn(2, 320, device=DEV, generator=gen).unbind(0)
    nv = torch.tensor([700], dtype=torch.int32, device=DEV)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(700, 320), dtype=torch.uint8, device=DEV)

    def outputs():
        return [torch.zeros(700, 320, dtype=BF16, device=DEV), torch.zeros(700, device=DEV),
                torch.zeros(700, device=DEV), torch.zeros(700, 320, dtype=BF16, device=DEV),
                torch.zeros(320, device=DEV), torch.zeros(320, device=DEV)]

    def run(o):
        B.ss_layernorm_rows_forward(x, nv, gamma, beta, EPS, o[0], o[1], o[2])
        B.ss_layernorm_rows_backward(dy, x, nv, gamma, o[1], o[2], o[3], o[4], o[5], ws)

    cap = outputs()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(cap)
    for n in (700, 699, 0, 333):
        nv.fill_(n)
        x.add_(0.25)
        eager = outputs()
        for o in cap:
            o.zero_()
        run(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, cap)), n


def test_offsets_beyond_32_bits():
    """Rows 2^29 + 1 elements apart: the later ones start beyond 2^32 bytes and 2^31 elements."""
    from paper_2404_04270_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(6)
    rows, dim, stride = 6, 5000, 2 ** 29 + 1
    wide = torch.empty(stride * (rows - 1) + dim, dtype=BF16, device=DEV)
    far = wide.as_strided((rows, dim), (stride, 1))
    x, dy = torch.randn(2, rows, dim, device=DEV, generator=gen).to(BF16).unbind(0)
    gamma, beta = torch.randn(2, dim, device=DEV, generator=gen).unbind(0)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)

    def out():
        return torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)

    near_y, mean, rstd = out()
    B.ss_layernorm_rows_forward(x, None, gamma, beta, EPS, near_y, mean, rstd)
    far.copy_(x)
    y, mean2, rstd2 = out()
    B.ss_layernorm_rows_forward(far, None, gamma, beta, EPS, y, mean2, rstd2)
    assert torch.equal(y, near_y) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    B.ss_layernorm_rows_forward(far, None, gamma, beta, EPS, far, mean2, rstd2)
    assert torch.equal(far, near_y)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
    B.ss_layernorm_rows_backward(dy, x, None, gamma, mean, rstd, dx, dg, db, ws)
    far.copy_(dy)
    dg2, db2 = torch.empty_like(gamma), torch.empty_like(gamma)
    B.ss_layernorm_rows_backward(far, x, None, gamma, mean, rstd, far, dg2, db2, ws)
    assert torch.equal(far, dx) and torch.equal(dg, dg2) and torch.equal(db, db2)


def test_refusals_of_the_python_calls():
    from paper_2404_04270_amd import binding as B
    x = torch.randn(4, 8, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    g = torch.ones(8, device=DEV)

    def forward(x=x, gamma=g, beta=g, y=y, mean=mean, rstd=rstd, eps=EPS, n_valid=None):
        B.ss_layernorm_rows_forward(x, n_valid, gamma, beta, eps, y, mean, rstd)

    forward()
    for bad in (dict(x=x.t()), dict(x=x[None]), dict(x=x.double()), dict(y=y.to(BF16)),
                dict(y=torch.empty(4, 9, device=DEV)), dict(gamma=g[:7]), dict(gamma=g.to(BF16)),
                dict(beta=g.double()), dict(gamma=torch.ones(16, device=DEV)[::2]),
                dict(mean=mean[:3]), dict(rstd=rstd.double()), dict(eps=-1.0),
                dict(x=x[:1].expand(4, 8)), dict(y=y.cpu()), dict(n_valid=torch.ones(1, device=DEV))):
        with pytest.raises(B.SlipstreamError):
            forward(**bad)
    with pytest.raises(B.SlipstreamError):               # parameters of two types
        forward(x=x.to(BF16), y=y.to(BF16), gamma=g, beta=g.to(BF16))
    with pytest.raises(B.SlipstreamError, match="workspace"):
        B.ss_layernorm_rows_backward(x, x, None, g, mean, rstd, y, g.clone(), None, None)
