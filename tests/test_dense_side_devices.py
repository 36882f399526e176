"""What the dense side's Python calls refuse by device and by length before the library is asked: no
kernel is launched (stand-ins for device tensors, at addresses that nothing reads)."""
import pytest
import torch

from paper_2404_04270_amd import binding as B
from test_sizes_beyond_32_bits import Stand, Stream, first_device  # noqa: F401


class On(Stand):
    def __init__(self, index, *args):
        super().__init__(*args)
        self.index, self.device = index, torch.device("cuda", index)

    def get_device(self):
        return self.index


def list_and_state(list_at, state_at):
    tensors, state = B.TensorList.__new__(B.TensorList), B.AdamWState.__new__(B.AdamWState)
    tensors.device, tensors.state_elems = torch.device("cuda", list_at), 128
    tensors.c = B._CTensorList(1, 1, 128, 4096)
    tensors.grads, tensors.only_grads = [], False
    tensors._pptr = tensors._gptr = On(list_at, torch.int64, 1)
    state.m = On(state_at, torch.uint8, 128)
    # (bits that the library refuses, should it be asked)
    state.c = B._CAdamWState(5, 0, 4096, 4096, 4096, None, 4096)
    return tensors, state


def test_moments_of_another_device():
    tensors, state = list_and_state(0, 1)
    out = On(0, torch.bfloat16, 128)
    with pytest.raises(B.SlipstreamError, match="another list"):
        B.ss_adamw_moments(tensors, state, out, out, Stream())
    with pytest.raises(B.SlipstreamError, match="another list"):
        B.ss_adamw_step(tensors, state, 1e-3, stream=Stream())
    tensors, state = list_and_state(0, 0)
    for wrong in (On(1, torch.bfloat16, 128), On(0, torch.bfloat16, 127), On(0, torch.float32, 128)):
        with pytest.raises(B.SlipstreamError, match="device 0|too small|dtype"):
            B.ss_adamw_moments(tensors, state, wrong, None, Stream())
    with pytest.raises(B.SlipstreamError, match="bits"):
        B.ss_adamw_moments(tensors, state, out, out, Stream())


def test_an_empty_count_of_valid_rows():
    """An empty tensor has no address, which the library takes for "all rows"."""
    x, per_row = On(0, torch.float32, 4, 8), On(0, torch.float32, 4)

    class Empty(Stand):
        def data_ptr(self):
            return 0

    none = Empty(torch.int32, 0)
    with pytest.raises(B.SlipstreamError, match="n_valid"):
        B.ss_layernorm_rows_forward(x, none, None, None, -1.0, x, per_row, per_row, Stream())
    with pytest.raises(B.SlipstreamError, match="n_valid"):
        B.ss_layernorm_rows_backward(x, x, none, None, per_row, per_row, x, On(0, torch.float32, 8),
                                     None, None, Stream())
