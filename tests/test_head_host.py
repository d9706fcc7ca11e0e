"""What the head's loss and the lists of tensors refuse, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2406_08334_amd import binding as B


def good(**kw):
    h = B.pt_head(0x1000, 0x2000, 0x3000, 0, 0x4000, 0, 0, 64, 64, 0, 0, 10, 100, 64, B.PT_BF16)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), B.PT_ERR_INVALID_ARG), (dict(vocab=0), B.PT_ERR_INVALID_ARG), (dict(width=0), B.PT_ERR_INVALID_ARG),
    (dict(weight=0), B.PT_ERR_INVALID_ARG), (dict(hidden=0), B.PT_ERR_INVALID_ARG), (dict(target=0), B.PT_ERR_INVALID_ARG),
    (dict(loss=0), B.PT_ERR_INVALID_ARG), (dict(hidden_stride=63), B.PT_ERR_INVALID_ARG), (dict(weight_stride=8), B.PT_ERR_INVALID_ARG),
    (dict(d_hidden=0x5000, d_hidden_stride=5), B.PT_ERR_INVALID_ARG), (dict(d_weight=0x5000, d_weight_stride=63), B.PT_ERR_INVALID_ARG),
    (dict(hidden=0x1001), B.PT_ERR_ALIGNMENT), (dict(row_scale=0x1002), B.PT_ERR_ALIGNMENT), (dict(target=0x1004), B.PT_ERR_ALIGNMENT),
    (dict(loss=0x1002), B.PT_ERR_ALIGNMENT), (dict(d_weight=0x5001, d_weight_stride=64), B.PT_ERR_ALIGNMENT),
    (dict(rows=(1 << 30) + 1), B.PT_ERR_UNSUPPORTED), (dict(vocab=(1 << 21) + 1), B.PT_ERR_UNSUPPORTED),
    (dict(width=(1 << 20) + 1, hidden_stride=1 << 21, weight_stride=1 << 21), B.PT_ERR_UNSUPPORTED),
    (dict(weight_stride=(1 << 21) + 8), B.PT_ERR_UNSUPPORTED)])
def test_a_head_that_is_refused(change, status):
    for fn in (lambda h: B.pt_head_workspace(h), lambda h: B.pt_head_loss(h, None, 0)):
        with pytest.raises(B.PtError) as e:
            fn(good(**change))
        assert e.value.status == status


def test_workspace_of_a_head():
    """Enough for what lies in it, growing with the rows up to a limit of pieces, and smaller without gradients."""
    least, best = B.pt_head_workspace(good())
    assert 0 < least <= best < 1 << 20
    assert B.pt_head_workspace(good(rows=0)) == (0, 0)
    big = dict(rows=16384, vocab=32000, width=4096, hidden_stride=4096, weight_stride=4096)
    loss_only = B.pt_head_workspace(good(**big))[1]
    least, best = B.pt_head_workspace(good(d_weight=0x5000, d_weight_stride=4096, **big))
    assert loss_only < least < best < 4 * 16384 * 32000           # less than the logits of all rows
    with pytest.raises(B.PtError) as e:
        B.pt_head_loss(good(**big), 0 or torch.empty(0, dtype=torch.uint8), 0)
    assert e.value.status == B.PT_ERR_INVALID_ARG
    L = B.lib()
    assert L.pt_head_workspace(None, None, None) == B.PT_ERR_INVALID_ARG
    assert L.pt_head_loss(None, None, 0, None) == B.PT_ERR_INVALID_ARG
    assert L.pt_head_workspace(C.byref(good()), None, None) == B.PT_OK


def test_what_the_helpers_refuse():
    h, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16)
    y, loss = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    assert B.head(h, w, y, loss).rows == 4
    assert B.head(h.t().contiguous().t()[:, :1], w[:, :1], y, loss).hidden_stride == 1
    for args in ((h.float(), w, y, loss), (h, w.half(), y, loss), (h, w[:, :7], y, loss), (h.t().contiguous().t(), w, y, loss),
                 (h, w, y.int(), loss), (h, w, y[:3], loss), (h, w, y, loss.double())):
        with pytest.raises(ValueError):
            B.head(*args)
    f = torch.zeros(300)
    c = torch.zeros(300, dtype=torch.uint8)
    assert B.tensor(f, f, f, f).flags == B.PT_TENSOR_GRAD_F32
    assert B.tensor(h.view(-1), f[:32], c[:32], c[:32], m_scale=f[:1], v_scale=f[:1], no_decay=True).flags == B.PT_TENSOR_NO_DECAY
    for kw in (dict(m=f[:299]), dict(m=c), dict(m=c, v=c, m_scale=f[:1], v_scale=f[:1]), dict(param16=f), dict(master=f.half()),
               dict(grad=torch.zeros(600)[::2])):
        with pytest.raises(ValueError):
            B.tensor(**{**dict(grad=f, master=f, m=f, v=f), **kw})


@pytest.mark.parametrize("change,status", [
    (dict(dtype=5), B.PT_ERR_INVALID_ARG), (dict(bits=16), B.PT_ERR_INVALID_ARG), (dict(grad=0), B.PT_ERR_INVALID_ARG),
    (dict(master=0), B.PT_ERR_INVALID_ARG), (dict(m=0), B.PT_ERR_INVALID_ARG), (dict(v=0), B.PT_ERR_INVALID_ARG),
    (dict(m_scale=0, bits=8), B.PT_ERR_INVALID_ARG), (dict(flags=4), B.PT_ERR_INVALID_ARG), (dict(grad=0x1001), B.PT_ERR_ALIGNMENT),
    (dict(grad=0x1002, flags=2), B.PT_ERR_ALIGNMENT), (dict(master=0x1002), B.PT_ERR_ALIGNMENT), (dict(m=0x1002, bits=8), B.PT_ERR_ALIGNMENT),
    (dict(param16=0x1001), B.PT_ERR_ALIGNMENT), (dict(elems=(1 << 40) + 1), B.PT_ERR_UNSUPPORTED), (dict(elems=1 << 40), B.PT_ERR_UNSUPPORTED),
    (dict(scaler=B.pt_scaler_cfg(0.5, 2.0, 0.5, 10, 0)), B.PT_ERR_INVALID_ARG)])
def test_a_list_that_is_refused(change, status):
    kw = dict(dtype=B.PT_BF16, bits=32, scaler=None)
    t = B.pt_tensor(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 100, 0, 0)
    for k, v in change.items():
        if k in kw:
            kw[k] = v
        else:
            setattr(t, k, v)
    with pytest.raises(B.PtError) as e:
        B.pt_tensors_create(kw["dtype"], [t], kw["bits"], kw["scaler"])
    assert e.value.status == status


def test_calls_without_a_list():
    L = B.lib()
    hp = B.hparams(1e-3, 0.9, 0.95, 1e-8, 0.1, 1.0)
    assert L.pt_tensors_destroy(None) == B.PT_OK
    assert L.pt_tensors_create(None, 0, None, 0, 32, None, 0) == B.PT_ERR_INVALID_ARG
    assert L.pt_tensors_create(C.byref(C.c_void_p()), 0, None, 1, 32, None, 0) == B.PT_ERR_INVALID_ARG
    assert L.pt_tensors_grad_sqnorm(None, None) == B.PT_ERR_INVALID_ARG
    assert L.pt_tensors_adamw_step(None, C.byref(hp), None) == B.PT_ERR_INVALID_ARG
    assert L.pt_tensors_set_state(None, 0, 1.0, 0, None) == B.PT_ERR_INVALID_ARG
    assert L.pt_tensors_report_read(None, None, None) == B.PT_ERR_INVALID_ARG
