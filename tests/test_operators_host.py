"""What the helpers and entry points of the head's loss and of lists of tensors refuse before anything reaches a device, and where their limits lie."""
import pytest
import torch

from paper_2406_08334_amd import binding as B
from test_head_host import good


def tensor8(grad_dtype=torch.bfloat16, param_dtype=torch.bfloat16):
    f, c = torch.zeros(300), torch.zeros(300, dtype=torch.uint8)
    return B.tensor(torch.zeros(300, dtype=grad_dtype), f, c, c.clone(), torch.zeros(300, dtype=param_dtype), m_scale=f[:2], v_scale=f[2:4])


def test_states_of_one_width_are_no_list_of_the_other():
    """Codes of a byte read and written as fp32 numbers would pass their arrays' ends."""
    f = torch.zeros(300)
    with pytest.raises(ValueError):
        B.pt_tensors_create(B.PT_BF16, [tensor8()], 32)
    with pytest.raises(ValueError):
        B.pt_tensors_create(B.PT_BF16, [B.tensor(f, f, f, f)], 8)
    with pytest.raises(ValueError):
        B.pt_tensors_create(B.PT_BF16, [B.tensor(f, f, f, f), tensor8()], 32)


@pytest.mark.parametrize("own,other", [((B.PT_BF16, torch.bfloat16), torch.float16), ((B.PT_FP16, torch.float16), torch.bfloat16)])
def test_arrays_of_the_other_16_bit_type(own, other):
    """Both have two bytes an element: read as the list's own they are other numbers."""
    for types in ((other, other), (own[1], other), (other, own[1])):
        with pytest.raises(ValueError):
            B.pt_tensors_create(own[0], [tensor8(*types)], 8)


@pytest.mark.parametrize("workspace", [torch.empty(1, dtype=torch.uint8).expand(1 << 24), torch.empty(1 << 16, 256, dtype=torch.uint8)[:, :128],
                                       torch.empty(1 << 24, dtype=torch.uint8)[::2]])
def test_a_workspace_with_gaps(workspace):
    """Its elements say nothing about the bytes behind its address: one byte expanded to 16 MiB passed for 16 MiB."""
    with pytest.raises(ValueError):
        B.pt_head_loss(good(), workspace, 0)


@pytest.mark.parametrize("limit,beyond", [(dict(rows=1 << 25), dict(rows=(1 << 25) + 1)),
                                          (dict(vocab=1 << 21), dict(vocab=(1 << 21) + 1)),
                                          (dict(width=1 << 20, hidden_stride=1 << 20, weight_stride=1 << 20),
                                           dict(width=(1 << 20) + 1, hidden_stride=1 << 21, weight_stride=1 << 21)),
                                          (dict(weight_stride=1 << 21), dict(weight_stride=(1 << 21) + 1))])
def test_the_limits_themselves(limit, beyond):
    """As the header names them: the last that is taken, the first that is not."""
    least, best = B.pt_head_workspace(good(**limit))
    assert 0 < least <= best
    for grads in (dict(d_hidden=0x10000, d_hidden_stride=1 << 21), dict(d_weight=0x20000, d_weight_stride=1 << 21)):
        least, best = B.pt_head_workspace(good(**limit, **grads))
        assert 0 < least <= best
        with pytest.raises(B.PtError) as e:
            B.pt_head_workspace(good(**beyond, **grads))
        assert e.value.status == B.PT_ERR_UNSUPPORTED
