"""What the layers before the head refuse, and what workspaces they ask for, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2406_08334_amd import binding as B

ARG, ALIGN, UNSUPPORTED, NOMEM = B.PT_ERR_INVALID_ARG, B.PT_ERR_ALIGNMENT, B.PT_ERR_UNSUPPORTED, B.PT_ERR_NOMEM


def made(struct, kw, change):
    s = struct(**kw)
    for k, v in change.items():
        if k in ("p", "step"):
            setattr(s.drop, k, v)
        else:
            setattr(s, k, v)
    return s


def refused(status, *calls):
    for f in calls:
        with pytest.raises(B.PtError) as e:
            f()
        assert e.value.status == status
        assert str(e.value)


LINEAR = dict(x=0x1000, weight=0x2000, out=0x3000, pre=0x4000, gate=0x5000, d_out=0x6000, d_x=0x7000, d_weight=0x8000, d_bias=0x9000, d_gate=0xa000, rows=100,
              outs=100, width=60, x_stride=64, weight_stride=64, gate_stride=100, residual_stride=100, pre_stride=100, out_stride=100, d_out_stride=100,
              d_x_stride=64, d_weight_stride=64, d_gate_stride=100, act=B.PT_ACT["silu"])


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), ARG), (dict(act=5), ARG), (dict(act=-1), ARG), (dict(outs=0), ARG), (dict(width=0), ARG), (dict(p=1.0), ARG), (dict(p=-0.1), ARG),
    (dict(p=float("nan")), ARG), (dict(x_scale=0x100), ARG), (dict(weight_scale=0x100), ARG), (dict(x_stride=59), ARG), (dict(weight_stride=1), ARG),
    (dict(gate_stride=99), ARG), (dict(residual=0x100, residual_stride=99), ARG), (dict(pre_stride=99), ARG), (dict(out_stride=99), ARG), (dict(d_out_stride=9), ARG),
    (dict(d_x_stride=59), ARG), (dict(d_weight_stride=59), ARG), (dict(d_gate_stride=0), ARG), (dict(x=0x1001), ALIGN), (dict(out=0x1001), ALIGN),
    (dict(bias=0x1001), ALIGN), (dict(d_bias=0x1001), ALIGN), (dict(step=0x1004), ALIGN), (dict(x_scale=0x1002, weight_scale=0x1000), ALIGN),
    (dict(rows=(1 << 25) + 1), UNSUPPORTED), (dict(outs=(1 << 21) + 1, **{k: 1 << 22 for k in LINEAR if k.endswith("_stride")}), UNSUPPORTED),
    (dict(width=(1 << 20) + 1, x_stride=1 << 21, weight_stride=1 << 21, d_x_stride=1 << 21, d_weight_stride=1 << 21), UNSUPPORTED),
    (dict(rows=1 << 25, outs=1 << 21, **{k: 1 << 22 for k in LINEAR if k.endswith("_stride")}), UNSUPPORTED)])
def test_a_layer_that_is_refused(change, status):
    d = made(B.pt_linear, LINEAR, change)
    refused(status, lambda: B.pt_linear_workspace(d), lambda: B.pt_linear_out(d, None, 0), lambda: B.pt_linear_grads(d, None, 0))


def test_what_each_call_of_a_layer_needs():
    out, grads = B.pt_linear_workspace(made(B.pt_linear, LINEAR, {}))
    assert out > 0 and grads > 0 and B.pt_linear_workspace(made(B.pt_linear, LINEAR, dict(rows=16)))[0] == 0      # few rows: none is needed
    room = torch.empty(1 << 20, dtype=torch.uint8)
    for change in (dict(x=0), dict(weight=0), dict(out=0)):
        refused(ARG, lambda: B.pt_linear_out(made(B.pt_linear, LINEAR, change), room, 0))
    for change in (dict(x=0), dict(weight=0), dict(pre=0), dict(d_out=0), dict(gate=0), dict(pre=0, act=0)):
        refused(ARG, lambda: B.pt_linear_grads(made(B.pt_linear, LINEAR, change), room, 0))
    refused(UNSUPPORTED, lambda: B.pt_linear_grads(made(B.pt_linear, LINEAR, dict(x_scale=0x100, weight_scale=0x200)), room, 0))
    L, d = B.lib(), made(B.pt_linear, LINEAR, {})
    for call, need in ((L.pt_linear_out, out), (L.pt_linear_grads, grads)):
        assert call(C.byref(d), None, need, None) == ARG
        assert call(C.byref(d), 0x1080, need, None) == ALIGN
        assert call(C.byref(d), 0x1000, need - 1, None) == NOMEM
        assert call(None, None, 0, None) == ARG
    assert L.pt_linear_workspace(None, None, None) == ARG and L.pt_linear_workspace(C.byref(d), None, None) == B.PT_OK
    assert B.pt_linear_workspace(made(B.pt_linear, LINEAR, dict(rows=0))) == (0, 0)
    assert B.pt_linear_out(made(B.pt_linear, LINEAR, dict(rows=0)), None, 0) is None


RMS = dict(x=0x1000, residual=0x2000, gain=0x3000, sum=0x4000, rstd=0x5000, y=0x6000, d_y=0x7000, d_sum=0x8000, d_x=0x9000, d_gain=0xa000, x_stride=100,
           residual_stride=100, sum_stride=100, y_stride=100, d_y_stride=100, d_sum_stride=100, d_x_stride=100, eps=1e-5, rows=10, width=100)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), ARG), (dict(width=0), ARG), (dict(eps=-1e-9), ARG), (dict(eps=float("nan")), ARG), (dict(x_stride=99), ARG), (dict(residual_stride=9), ARG),
    (dict(sum_stride=9), ARG), (dict(y_stride=9), ARG), (dict(d_y_stride=9), ARG), (dict(d_sum_stride=9), ARG), (dict(d_x_stride=9), ARG), (dict(x=0x1001), ALIGN),
    (dict(y=0x1001), ALIGN), (dict(gain=0x1001), ALIGN), (dict(d_gain=0x1001), ALIGN), (dict(rstd=0x1002), ALIGN), (dict(y_scale=0x1002), ALIGN),
    (dict(rows=(1 << 30) + 1), UNSUPPORTED), (dict(width=32769, **{k: 40000 for k in RMS if k.endswith("_stride")}), UNSUPPORTED)])
def test_a_norm_that_is_refused(change, status):
    d = made(B.pt_rms, RMS, change)
    refused(status, lambda: B.pt_rms_workspace(d), lambda: B.pt_rms_norm(d, 0), lambda: B.pt_rms_grads(d, None, 0))


def test_what_each_call_of_a_norm_needs():
    need = B.pt_rms_workspace(made(B.pt_rms, RMS, {}))
    assert need > 0 and B.pt_rms_workspace(made(B.pt_rms, RMS, dict(d_gain=0))) == 0
    for change in (dict(x=0), dict(y=0)):
        refused(ARG, lambda: B.pt_rms_norm(made(B.pt_rms, RMS, change), 0))
    room = torch.empty(1 << 20, dtype=torch.uint8)
    for change in (dict(sum=0), dict(sum=0, x=0, residual=0), dict(rstd=0), dict(d_y=0)):
        refused(ARG, lambda: B.pt_rms_grads(made(B.pt_rms, RMS, change), room, 0))
    L, d = B.lib(), made(B.pt_rms, RMS, {})
    assert L.pt_rms_grads(C.byref(d), None, need, None) == ARG
    assert L.pt_rms_grads(C.byref(d), 0x1080, need, None) == ALIGN
    assert L.pt_rms_grads(C.byref(d), 0x1000, need - 1, None) == NOMEM
    assert L.pt_rms_norm(None, None) == ARG and L.pt_rms_grads(None, None, 0, None) == ARG and L.pt_rms_workspace(None, None) == ARG
    assert B.pt_rms_norm(made(B.pt_rms, RMS, dict(rows=0)), 0) is None
    assert B.pt_rms_grads(made(B.pt_rms, RMS, dict(d_x=0, d_gain=0)), None, 0) is None


ROWS = dict(x=0x1000, codes=0x2001, scale=0x3000, x_stride=100, codes_stride=100, rows=10, width=100)


@pytest.mark.parametrize("change,status", [
    (dict(type=3), ARG), (dict(width=0), ARG), (dict(x=0), ARG), (dict(codes=0), ARG), (dict(scale=0), ARG), (dict(x_stride=99), ARG), (dict(codes_stride=99), ARG),
    (dict(x=0x1001), ALIGN), (dict(x=0x1002, type=B.PT_FP32), ALIGN), (dict(scale=0x1001), ALIGN),
    (dict(width=32769, x_stride=40000, codes_stride=40000), UNSUPPORTED), (dict(rows=(1 << 30) + 1), UNSUPPORTED)])
def test_rows_that_are_refused(change, status):
    refused(status, lambda: B.pt_rows8(made(B.pt_rows, ROWS, change), 0))


DROPPED = dict(x=0x1000, out=0x2000, x_stride=100, residual_stride=100, out_stride=100, rows=10, width=100)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), ARG), (dict(width=0), ARG), (dict(p=1.0), ARG), (dict(p=-1e-9), ARG), (dict(p=float("nan")), ARG), (dict(x=0), ARG), (dict(out=0), ARG),
    (dict(x_stride=99), ARG), (dict(out_stride=99), ARG), (dict(residual=0x100, residual_stride=99), ARG), (dict(x=0x1001), ALIGN), (dict(residual=0x101), ALIGN),
    (dict(step=0x1004), ALIGN), (dict(rows=(1 << 32) - 1), UNSUPPORTED)])
def test_dropout_that_is_refused(change, status):
    refused(status, lambda: B.pt_dropout(made(B.pt_dropped, DROPPED, change), 0))


def test_calls_without_a_description():
    L = B.lib()
    assert L.pt_rows8(None, None) == ARG and L.pt_dropout(None, None) == ARG
    assert B.pt_rows8(made(B.pt_rows, ROWS, dict(rows=0)), 0) is None and B.pt_dropout(made(B.pt_dropped, DROPPED, dict(rows=0)), 0) is None


def test_what_the_helpers_refuse():
    x, w, o = torch.zeros(4, 8).bfloat16(), torch.zeros(5, 8).bfloat16(), torch.zeros(4, 5).bfloat16()
    f, b = torch.zeros(4), torch.zeros(5).bfloat16()
    c = torch.zeros(4, 8, dtype=torch.uint8)
    assert B.linear(x, w, o, bias=b, act="gelu", drop=0.1, seed=-1).outs == 5
    assert B.linear(c, c[:3], o[:, :3], x_scale=f, weight_scale=f[:3]).dtype == B.PT_BF16
    assert B.linear(c, c[:3], o[:, :3].half(), x_scale=f, weight_scale=f[:3]).dtype == B.PT_FP16
    for args, kw in (((x.float(), w, o), {}), ((x, w.half(), o), {}), ((x, w[:, :7], o), {}), ((x, w, o.t()), {}), ((x, w, o), dict(bias=f)), ((x, w, o), dict(bias=b[:4])),
                     ((x, w, o), dict(gate=o[:3])), ((x, w, o), dict(act="tanh")), ((x, w, o), dict(step=f)), ((c, w, o), dict(x_scale=f, weight_scale=f)),
                     ((c, c[:3], o), dict(x_scale=f)), ((x, w, o), dict(d_x=o)), ((x, w, o), dict(x_scale=f, weight_scale=f)),
                     ((x.t().contiguous().t(), w, o), {})):
        with pytest.raises(ValueError):
            B.linear(*args, **kw)
    assert B.rms(x, x, gain=x[0]).width == 8
    assert B.rms(x, c, y_scale=f).y_stride == 8
    for args, kw in (((x.float(), x), {}), ((x, c), {}), ((x, x), dict(y_scale=f)), ((x, x), dict(gain=b)), ((x, x), dict(rstd=x[:, 0])), ((x, x), dict(residual=w)),
                     ((x, x), dict(d_gain=x[0].half()))):
        with pytest.raises(ValueError):
            B.rms(*args, **kw)
    assert B.rows8(x.float(), c, f).type == B.PT_FP32
    for args in ((x.double(), c, f), (x, x, f), (x, c[:3], f), (x, c, x[:, 0])):
        with pytest.raises(ValueError):
            B.rows8(*args)
    assert B.dropout(x, x, 0.5, 2 ** 64 + 3).drop.seed == 3
    for args, kw in (((x.float(), x, 0.1, 0), {}), ((x, o, 0.1, 0), {}), ((x, x, 0.1, 0), dict(residual=x.half())), ((x, x, 0.1, 0), dict(step=f[:1]))):
        with pytest.raises(ValueError):
            B.dropout(*args, **kw)
