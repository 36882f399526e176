"""Numbers that the C calls take in 32 bits are refused where they do not fit: cut to 32 bits they
would stand for a smaller matrix, of which a part would be worked on without a word.  No kernel is
launched: the tensors are stand-ins with a shape, and eps is one that the library refuses."""
import pytest
import torch

from paper_2404_04270_amd import binding as B

FAR = 1 << 32


class Stand:
    """What the calls ask of a contiguous device tensor, at an address that nothing reads."""

    def __init__(self, dtype, *shape):
        self.dtype, self.shape = dtype, torch.Size(shape)
        self.device, self.is_cuda = torch.device("cuda", 0), True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


class Stream:
    cuda_stream = 0


@pytest.fixture(autouse=True)
def first_device(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)


TOO_LARGE = [(FAR + 8, 1), (FAR + 8, 64), (5, FAR + 64), (FAR, 16), (1 << 31, 16), (3, 1 << 31)]


@pytest.mark.parametrize("rows,dim", TOO_LARGE)
def test_layernorm_rows_refuses_rows_and_columns_beyond_32_bits(rows, dim):
    bf, f = torch.bfloat16, torch.float32
    x, per_row, per_column = Stand(bf, rows, dim), Stand(f, rows), Stand(f, dim)
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.ss_layernorm_rows_forward(x, None, per_column, per_column, -1.0, x, per_row, per_row,
                                    Stream())
    # (without a workspace the library refuses the gradients of the parameters)
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.ss_layernorm_rows_backward(x, x, None, per_column, per_row, per_row, x, per_column, None,
                                     None, Stream())
    assert B.ss_layernorm_rows_workspace_bytes(rows, dim) == 0


def test_layernorm_rows_takes_what_fits():
    """The largest numbers get as far as the library's own checks."""
    f = torch.float32
    x, per_row = Stand(f, (1 << 31) - 1, 4), Stand(f, (1 << 31) - 1)
    with pytest.raises(B.SlipstreamError, match="eps"):
        B.ss_layernorm_rows_forward(x, None, None, None, -1.0, x, per_row, per_row, Stream())
    assert B.ss_layernorm_rows_workspace_bytes((1 << 31) - 1, 1) > 0
    assert B.ss_layernorm_rows_workspace_bytes(8, 1 << 20) > 0


class Tables(B.Tables):
    """Tables of stand-ins: the calls below end before anything reads a pointer."""

    def __init__(self, num_tables=1, rows=100, dim=4):
        self.num_tables, self.rows, self.dim = num_tables, rows, dim
        self.device = torch.device("cuda", 0)
        self._wptr, self._bptr = Stand(torch.int64, num_tables), None
        self._refresh_struct()


class Hot:
    def __init__(self, h=8):
        self.hot_ids, self.H = [Stand(torch.int32, h)], h
        self.drift = self.stale_hot = [Stand(torch.float64, h)]
        self._hptr = self._sptr = self._dptr = self._shptr = Stand(torch.int64, 1)
        self.stale_count = None


I32, F, U8 = torch.int32, torch.float32, torch.uint8
LARGE = 1 << 50                          # as many elements as any check asks for


def calls(b, l):
    """Every call that takes a batch's shape, of b samples with l lookups."""
    t, s = Tables(), Stream()
    idx, out, ws, i32 = Stand(I32, 1, b, l), Stand(F, LARGE), Stand(U8, LARGE), Stand(I32, LARGE)
    u8, y, per_row = Stand(U8, LARGE), Stand(F, 1, b, 4), Stand(F, LARGE)
    c = B.AccessCounters.__new__(B.AccessCounters)
    c.rows, c.counts, c._cptr = 100, [i32], Stand(torch.int64, 1)
    return {
        "ss_check_indices": lambda: B.ss_check_indices(1, 100, idx, None, Stand(torch.int64, 2), s),
        "ss_filter_batch": lambda: B.ss_filter_batch(t, idx, 1, u8, i32, i32, i32, ws, s),
        "ss_filter_batch_split": lambda: B.ss_filter_batch_split(t, None, idx, 1, u8, u8, i32, i32,
                                                                 i32, ws, s),
        "ss_embbag_forward": lambda: B.ss_embbag_forward(t, idx, None, out, s),
        "ss_embbag_backward_update": lambda: B.ss_embbag_backward_update(t, idx, None, out, 0.1, ws,
                                                                         s),
        "ss_embbag_backward_update_noalloc": lambda: B.ss_embbag_backward_update_noalloc(
            t, idx, None, out, 0.1, s),
        "ss_embbag_backward_prepare": lambda: B.ss_embbag_backward_prepare(t, idx, None, ws, s),
        "ss_embbag_forward_grouped": lambda: B.ss_embbag_forward_grouped(t, idx, None, out, ws, s),
        "ss_embbag_backward_apply": lambda: B.ss_embbag_backward_apply(t, b, l, out, 0.1, ws, s),
        "ss_embbag_forward_ln": lambda: B.ss_embbag_forward_ln(t, idx, None, None, None, 1e-5, y,
                                                               per_row, per_row, s),
        "ss_embbag_ln_backward": lambda: B.ss_embbag_ln_backward(t, idx, None, y, None, per_row,
                                                                 per_row, y, None, None, None, s),
        "ss_sample_drop": lambda: B.ss_sample_drop(Hot(), idx, 1, [0.5], i32, s),
        "ss_sample_levels": lambda: B.ss_sample_levels(Hot(), idx, Stand(F, b), s),
        "ss_count_accesses": lambda: B.ss_count_accesses(c, idx, None, s),
        "ss_step_plan_for": lambda: B.ss_step_plan_for(1, b, l),
    }


@pytest.mark.parametrize("b,l", [(FAR + 8, 1), (8, FAR + 1), (1 << 31, 2)])
@pytest.mark.parametrize("call", sorted(calls(1, 1)))
def test_batches_beyond_32_bits(call, b, l):
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        calls(b, l)[call]()


def test_other_sizes_beyond_32_bits():
    s, n = Stream(), FAR + 8
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.ss_level_counts(Stand(F, n), [0.5], Stand(I32, 4), s)
    x = Stand(F, 1, n, 64)
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.ss_layernorm_forward(x, None, None, None, 1e-5, x, Stand(F, n), Stand(F, n), s)
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.ss_layernorm_backward(x, x, None, None, Stand(F, n), Stand(F, n), x, None, None, None, s)
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.Tables([Stand(F, 2, FAR + 64)])
    for f in (B.ss_filter_batch_workspace_bytes, B.ss_layernorm_backward_workspace_bytes):
        assert f(1, FAR + 8, 4) == 0 and f(1, 8, FAR + 4) == 0
    assert B.ss_backward_workspace_bytes(1, FAR + 8, 1, 64) == 0
    assert B.ss_backward_workspace_bytes(1, 8, 1, FAR + 64) == 0


def test_hot_sets_beyond_32_bits():
    s, n = Stream(), FAR + 8
    c = B.AccessCounters.__new__(B.AccessCounters)
    c.rows, c.counts, c._cptr = 100, [Stand(I32, 100)], Stand(torch.int64, 1)
    c.device = torch.device("cuda", 0)
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.ss_select_hot_ratio(c, 0.1, 10, [Stand(I32, n)], None, None, Stand(U8, LARGE), s)
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.ss_select_hot_top(c, n, [Stand(I32, n)], None, Stand(U8, LARGE), s)
    with pytest.raises(B.SlipstreamError, match="beyond 32 bits"):
        B.HotState(Tables(), [Stand(I32, n)])
