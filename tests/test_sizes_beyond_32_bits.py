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
