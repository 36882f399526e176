"""The dense side's calls refuse what they cannot take, on the host: no kernel is launched."""
import ctypes as C
import math

import pytest

from paper_2404_04270_amd import binding as B

FAKE = 4096                     # an aligned address that no call below gets to use
lib = B._lib


def plan(tensors, size=None):
    arr = (B._CTensor * max(1, len(tensors)))(*tensors)
    out = B._CTensorList()
    rc = lib.ss_tensor_list_plan(arr, len(tensors), out, None, 0)
    return rc, out, arr


def test_plan_counts_chunks_and_pads_to_blocks():
    rc, out, arr = plan([(1, 0, 0, 0, 0), (0, 1, 1, 0, 0), (129, 2, 0, 1, 0), (100_000, 1, 0, 0, 0)])
    assert rc == 0 and out.num_tensors == 4
    assert out.state_elems == 128 + 0 + 256 + 100_096
    buf = C.create_string_buffer(out.num_chunks * 32)
    assert lib.ss_tensor_list_plan(arr, 4, out, C.addressof(buf), len(buf)) == 0
    import struct
    seen = {}
    for k in range(out.num_chunks):
        state, first, tensor, count, kind, _ = struct.unpack_from("<qqiiii", buf, 32 * k)
        assert count > 0 and first == seen.get(tensor, 0)
        assert state == {0: 0, 2: 128, 3: 384}[tensor] + first
        assert kind == {0: 0, 2: 2 | 16, 3: 1}[tensor]
        assert first % 128 == 0
        seen[tensor] = first + count
    assert seen == {0: 1, 2: 129, 3: 100_000}
    assert lib.ss_tensor_list_plan(arr, 4, out, C.addressof(buf), len(buf) - 1) == 3
    assert plan([])[0] == 0


@pytest.mark.parametrize("tensor,text", [
    ((-1, 0, 0, 0, 0), "numel"), ((1 << 47, 0, 0, 0, 0), "numel"), ((5, 3, 3, 0, 0), "dtype"),
    ((5, -1, 0, 0, 0), "dtype"), ((5, 0, 1, 0, 0), "grad_dtype"), ((5, 1, 2, 0, 0), "grad_dtype"),
    ((5, 1, 1, 2, 0), "no_decay"), ((5, 1, 1, 0, 9), "reserved")])
def test_plan_refuses(tensor, text):
    rc, _, _ = plan([(1, 0, 0, 0, 0), tensor])
    assert rc == 1 and text in B.ss_last_error()


def test_plan_refuses_a_list_that_is_too_long():
    rc, out, _ = plan([((1 << 24) * 2048 - 2048, 1, 1, 0, 0)])
    assert rc == 0 and out.num_chunks == (1 << 24) - 1
    rc, _, _ = plan([((1 << 24) * 2048 - 2048, 1, 1, 0, 0), (1, 0, 0, 0, 0)])
    assert rc == 2 and "too long" in B.ss_last_error()


def a_list(chunks=3):
    return B._CTensorList(1, chunks, 8192 * chunks, FAKE)


@pytest.mark.parametrize("change,text", [
    (dict(lst=None), "list is NULL"), (dict(lst=B._CTensorList(1, 3, 1, None)), "chunks"),
    (dict(lst=B._CTensorList(1, -3, 1, FAKE)), "planned"), (dict(grads=None), "NULL"),
    (dict(lst=B._CTensorList(1, 3, 1, FAKE + 4)), "aligned"),
    (dict(clip=None), "NULL"), (dict(clip=FAKE + 4), "aligned"), (dict(max_norm=0.0), "max_norm"),
    (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=math.nan), "max_norm"),
    (dict(scale=math.inf), "grad_scale"), (dict(scale=math.nan), "grad_scale"),
    (dict(ws=None), "workspace"), (dict(ws=FAKE + 8), "workspace"), (dict(size=8), "workspace")])
def test_grad_norm_refuses(change, text):
    a = dict(lst=a_list(), grads=FAKE, max_norm=1.0, scale=1.0, clip=FAKE, ws=FAKE, size=1 << 20)
    a.update(change)
    rc = lib.ss_grad_norm(a["lst"], a["grads"], a["max_norm"], a["scale"], a["clip"], a["ws"],
                          a["size"], None)
    assert rc != 0 and text in B.ss_last_error()


def state(**kw):
    a = dict(bits=32, m=FAKE, v=FAKE, exps=None, master=None, counters=FAKE)
    a.update(kw)
    return B._CAdamWState(a["bits"], 0, a["m"], a["v"], a["exps"], a["master"], a["counters"])


@pytest.mark.parametrize("change,text", [
    (dict(lst=None), "list is NULL"), (dict(params=None), "NULL"), (dict(grads=None), "NULL"),
    (dict(state=None), "state is NULL"),
    (dict(state=state(bits=16)), "bits"), (dict(state=state(m=None)), "NULL"),
    (dict(state=state(bits=8)), "exps"), (dict(state=state(v=FAKE + 8)), "aligned"),
    (dict(state=state(master=FAKE + 4)), "master"), (dict(state=state(counters=None)), "counters"),
    (dict(state=state(counters=FAKE + 16)), "counters"), (dict(clip=FAKE + 8), "clip"),
    (dict(lr=-1.0), "lr"), (dict(lr=math.nan), "lr"),
    (dict(weight_decay=-0.1), "weight_decay"),
    (dict(beta1=1.0), "beta1"), (dict(beta2=-0.1), "beta2"),
    (dict(beta2=math.nan), "beta2"), (dict(eps=0.0), "eps"),
    (dict(eps=math.inf), "eps")])
def test_adamw_step_refuses(change, text):
    a = dict(lst=a_list(), params=FAKE, grads=FAKE, state=state(), lr=1e-3, beta1=0.9, beta2=0.999,
             eps=1e-8, weight_decay=0.01, clip=None)
    a.update(change)
    rc = lib.ss_adamw_step(a["lst"], a["params"], a["grads"], a["state"], a["lr"], None, a["beta1"],
                           a["beta2"], a["eps"], a["weight_decay"], a["clip"], None)
    assert rc == 1 and text in B.ss_last_error()


def test_moments_refuses_32_bits_and_places_of_no_bf16_vector():
    assert lib.ss_adamw_moments(a_list(), state(), FAKE, FAKE, None) == 1
    assert "32 bits" in B.ss_last_error()
    assert lib.ss_adamw_moments(a_list(), state(bits=8, exps=FAKE), FAKE + 2, None, None) == 1
    assert "aligned" in B.ss_last_error()


ROWS = dict(dtype=1, param=0, rows=8, dim=100, x=FAKE, xs=100, nv=None, gamma=FAKE, beta=FAKE,
            eps=1e-5, y=FAKE, ys=100, mean=FAKE, rstd=FAKE)


@pytest.mark.parametrize("change,text", [
    (dict(dtype=3), "dtype"), (dict(param=2), "param_dtype"), (dict(rows=-1), "rows"),
    (dict(dim=0), "dim"), (dict(dim=(1 << 20) + 1), "dim"), (dict(x=None), "x is NULL"),
    (dict(y=None), "y is NULL"), (dict(xs=99), "apart"), (dict(ys=99), "apart"),
    (dict(x=FAKE + 1), "aligned"), (dict(gamma=FAKE + 2), "gamma"), (dict(mean=None), "mean"),
    (dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"), (dict(ys=101), "another stride")])
def test_layernorm_rows_forward_refuses(change, text):
    a = dict(ROWS, **change)
    rc = lib.ss_layernorm_rows_forward(
        a["dtype"], a["param"], a["rows"], a["dim"], a["x"], a["xs"], a["nv"], a["gamma"],
        a["beta"], a["eps"], a["y"], a["ys"], a["mean"], a["rstd"], None)
    assert rc == 1 and text in B.ss_last_error()


@pytest.mark.parametrize("change,text", [
    (dict(dtype=-1), "dtype"), (dict(param=2), "param_dtype"), (dict(dy=None), "dy is NULL"),
    (dict(dx=FAKE + 1), "dx"), (dict(dys=99), "apart"), (dict(dxs=101), "another stride"),
    (dict(rstd=None), "rstd"), (dict(ws=None), "workspace"), (dict(ws=FAKE + 16), "workspace"),
    (dict(size=100), "workspace"), (dict(dgamma=FAKE + 2), "dgamma")])
def test_layernorm_rows_backward_refuses(change, text):
    a = dict(ROWS, dy=FAKE, dys=100, dx=FAKE, dxs=100, dgamma=FAKE, dbeta=FAKE, ws=FAKE, size=1 << 20)
    a.update(change)
    rc = lib.ss_layernorm_rows_backward(
        a["dtype"], a["param"], a["rows"], a["dim"], a["dy"], a["dys"], a["x"], a["xs"], a["nv"],
        a["gamma"], a["mean"], a["rstd"], a["dx"], a["dxs"], a["dgamma"], a["dbeta"], a["ws"],
        a["size"], None)
    assert rc in (1, 3) and text in B.ss_last_error()


def test_rows_workspace_falls_in_neither_argument():
    last = 0
    rows = [0, 1, 2, 5, 17, 100, 1023, 1024, 1025, 5000, 1 << 20]
    dims = [1, 2, 63, 64, 1000, 4095, 4096, 4097, 8192, 16385, 100_000, 262_144, 262_145, 1 << 20]
    for d in dims:
        for a, b in zip(rows, rows[1:]):
            assert B.ss_layernorm_rows_workspace_bytes(a, d) <= B.ss_layernorm_rows_workspace_bytes(b, d)
    for r in rows:
        for a, b in zip(dims, dims[1:]):
            last = B.ss_layernorm_rows_workspace_bytes(r, a)
            assert 0 < last <= B.ss_layernorm_rows_workspace_bytes(r, b), (r, a, b)
    assert B.ss_layernorm_rows_workspace_bytes(5, 0) == 0
    assert B.ss_layernorm_rows_workspace_bytes(-1, 5) == 0


def test_python_calls_refuse_host_tensors_and_wrong_types():
    import torch
    with pytest.raises(B.SlipstreamError):
        B.TensorList([])
    with pytest.raises(B.SlipstreamError):
        B.TensorList([torch.zeros(4)])
    with pytest.raises(B.SlipstreamError):
        B.TensorList([torch.zeros(4, dtype=torch.float64)])
    x = torch.zeros(4, 8)
    with pytest.raises(B.SlipstreamError):
        B.ss_layernorm_rows_forward(x, None, None, None, 1e-5, x, x[0], x[0])
