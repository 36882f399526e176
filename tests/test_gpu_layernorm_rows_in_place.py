"""LayerNorm of rows in place (y is x; dx is dy or x) gives the bits of the same call into a matrix of
its own, for every group of lanes, rows that end inside a vector (whose last vector is read shifted
back over columns that another lane stores) and so many rows that every group takes several."""
import pytest
import torch

from test_gpu_layernorm_rows import BF16, DEV, EPS, F16, F32, matrix

pytestmark = pytest.mark.gpu

# rows beyond one turn of the grid: 131072 in 2 lanes, 4096 in 64, 1024 in 256, 512 in 512, 1024 where a
# row does not fit a workgroup's registers
SHAPES = [(140_001, 13), (9001, 301), (9001, 1001), (2300, 1999), (2300, 3001), (1300, 6001),
          (1300, 9001), (1300, 16_383), (1100, 50_001)]


def case(rows, dim, dtype, wt, pad, n_valid):
    from paper_2404_04270_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(rows + dim)
    nv = None if n_valid is None else torch.tensor([n_valid], dtype=torch.int32, device=DEV)
    gamma = (torch.randn(dim, device=DEV, generator=gen) * 0.2 + 1).to(wt)
    beta = (torch.randn(dim, device=DEV, generator=gen) * 0.2).to(wt)
    xbuf, x = matrix(rows, dim, dtype, gen, pad)
    dbuf, dy = matrix(rows, dim, dtype, gen, pad, shift=0.1, scale=0.5)
    ws = torch.empty(B.ss_layernorm_rows_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)

    def copy(buf):
        buf = buf.clone()
        return buf, buf[1:].view(rows, dim + pad)[:, :dim]

    def stats():
        return torch.zeros(2, rows, device=DEV).unbind(0)

    ybuf, y = copy(xbuf)
    mean, rstd = stats()
    B.ss_layernorm_rows_forward(x, nv, gamma, beta, EPS, y, mean, rstd)
    zbuf, z = copy(xbuf)
    mean2, rstd2 = stats()
    B.ss_layernorm_rows_forward(z, nv, gamma, beta, EPS, z, mean2, rstd2)
    assert torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    assert torch.equal(ybuf, zbuf)           # rows that do not count and what lies between, too
    del ybuf, y, zbuf, z

    for source in ("dy", "x"):
        obuf, out = copy(dbuf if source == "dy" else xbuf)
        dg, db = torch.empty(2, dim, device=DEV).to(wt).unbind(0)
        B.ss_layernorm_rows_backward(dy, x, nv, gamma, mean, rstd, out, dg, db, ws)
        a, b = copy(dbuf), copy(xbuf)
        dg2, db2 = torch.empty(2, dim, device=DEV).to(wt).unbind(0)
        over = a if source == "dy" else b
        B.ss_layernorm_rows_backward(a[1], b[1], nv, gamma, mean, rstd, over[1], dg2, db2, ws)
        assert torch.equal(over[0], obuf), source
        assert torch.equal(dg, dg2) and torch.equal(db, db2), source
        # without the parameters' gradients: the same dx
        c, d = copy(dbuf), copy(xbuf)
        over = c if source == "dy" else d
        B.ss_layernorm_rows_backward(c[1], d[1], nv, gamma, mean, rstd, over[1], None, None, None)
        assert torch.equal(over[0], obuf), source


@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("dtype,wt", [(F32, F32), (BF16, F32), (F16, F16)])
def test_in_place_gives_the_same_bits(rows, dim, dtype, wt):
    case(rows, dim, dtype, wt, pad=3, n_valid=rows - 1)


@pytest.mark.parametrize("rows,dim,dtype,wt,pad", [
    # results past the caches (rows at even places), inputs past them
    (4200, 16_383, F32, F32, 1), (9000, 8191, BF16, BF16, 1), (2200, 16_381, BF16, F32, 3),
    # few rows: one workgroup takes them all
    (4, 9001, F16, F16, 0), (4, 16_383, F32, F32, 5), (8, 3001, BF16, BF16, 0), (32, 1001, F16, F32, 7)])
def test_in_place_past_the_caches_and_in_one_workgroup(rows, dim, dtype, wt, pad):
    case(rows, dim, dtype, wt, pad, None)
