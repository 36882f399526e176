"""What lies in the master copies of a list of several types."""
import pytest
import torch

from test_gpu_adamw import F32
from test_gpu_adamw_mixed import mixed_list

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_master_copies_are_of_16_bit_parameters_only(bits):
    """The places of fp32 tensors hold 0, before and after steps: a copy that no step keeps up would
    be an old value to whoever reads or restores it."""
    opt, params, _ = mixed_list(True, state_bits=bits)
    for _ in range(3):
        for k, p in enumerate(params):
            copy = opt.list.of(opt.state.master, k)
            if p.dtype is F32:
                assert not bool(copy.any()), k
            else:
                assert torch.equal(p, copy.to(p.dtype)), k
        opt.step()
