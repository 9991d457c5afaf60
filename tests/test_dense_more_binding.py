"""The gated block's, the cross entropy's and AdamW's binding against their header, and their refusals, without a GPU."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2504_01506_gb300 import _lib, build, dense

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mlkv_dense.h")
P = 4096  # a pointer that no call here reads


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


@pytest.mark.parametrize("name,struct", [("mlkv_gated_linear_args", _lib.GatedLinearArgs), ("mlkv_linear_cross_entropy_args", _lib.LinearCrossEntropyArgs),
                                         ("mlkv_adamw_tensor", _lib.AdamWTensor), ("mlkv_adamw_args", _lib.AdamWArgs)])
def test_argument_structs_match_the_header(name, struct, tmp_path):
    fields = [f for f, _ in struct._fields_]
    prog = tmp_path / "layout.c"
    body = "".join(f'printf("{f} %zu\\n", offsetof({name}, {f}));' for f in fields)
    prog.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mlkv_dense.h"\n'
                    f'int main(void){{printf("size %zu\\n", sizeof({name}));{body}return 0;}}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.dirname(HEADER), str(prog), "-o", str(exe)], check=True)
    out = dict(ln.split() for ln in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(out["size"]) == ctypes.sizeof(struct)
    for f in fields:
        assert int(out[f]) == getattr(struct, f).offset, f


def test_gated_linear_refusals(lib):
    good = dict(m=4, f=8, k=8, d_x=P, x_stride=8, d_w_gate=P, w_gate_stride=8, d_w_up=P, w_up_stride=8, d_h=P, h_stride=8, type=_lib.TYPE_BFLOAT,
                activation=_lib.ACT_SILU)
    bads = (dict(m=-1), dict(f=-1), dict(k=-1), dict(m=2 ** 29), dict(f=2 ** 29), dict(type=_lib.TYPE_FLOAT), dict(type=7), dict(activation=4),
            dict(activation=-1), dict(d_x=None), dict(x_stride=7), dict(d_w_gate=None), dict(w_gate_stride=7), dict(d_w_up=None), dict(w_up_stride=2 ** 38))
    for bad in (*bads, dict(d_h=None), dict(h_stride=7), dict(d_gate=P, gate_stride=8), dict(d_up=P, up_stride=8),
                dict(d_gate=P, gate_stride=7, d_up=P, up_stride=8)):
        a = _lib.GatedLinearArgs(**{**good, **bad})
        assert lib.mlkv_gated_linear(a, None) == _lib.ERR_INVALID, bad
        assert lib.mlkv_gated_linear_workspace(a) == -1
    good.update(d_dh=P, dh_stride=8, d_gate=P, gate_stride=8, d_up=P, up_stride=8, d_dx=P, dx_stride=8, d_dw_gate=P, dw_gate_stride=8, d_dw_up=P, dw_up_stride=8)
    for bad in (*bads, dict(d_dh=None), dict(dh_stride=7), dict(d_gate=None), dict(d_up=None), dict(up_stride=2), dict(dx_stride=7), dict(dw_gate_stride=7),
                dict(dw_up_stride=1)):
        a = _lib.GatedLinearArgs(**{**good, **bad})
        assert lib.mlkv_gated_linear_backward(a, None) == _lib.ERR_INVALID, bad
        assert lib.mlkv_gated_linear_backward_workspace(a) == -1
    assert lib.mlkv_gated_linear(None, None) == _lib.ERR_INVALID


def test_linear_cross_entropy_refusals(lib):
    good = dict(n=4, k=8, vocab=16, d_x=P, x_stride=8, d_weight=P, weight_stride=8, d_targets=P, d_loss=P, d_stats=P, scale=1.0, type=_lib.TYPE_HALF)
    bads = (dict(n=-1), dict(k=0), dict(vocab=0), dict(n=2 ** 30), dict(vocab=2 ** 30), dict(type=_lib.TYPE_FLOAT), dict(scale=0.0), dict(scale=-1.0),
            dict(scale=math.inf), dict(scale=2.0 ** 127), dict(scale=math.nan), dict(d_x=None), dict(x_stride=7), dict(d_weight=None), dict(weight_stride=7), dict(d_targets=None),
            dict(d_stats=None))
    for bad in (*bads, dict(d_loss=None)):
        a = _lib.LinearCrossEntropyArgs(**{**good, **bad})
        assert lib.mlkv_linear_cross_entropy(a, None) == _lib.ERR_INVALID, bad
        assert lib.mlkv_linear_cross_entropy_workspace(a) == -1
    good.update(d_dloss=P, d_dx=P, dx_stride=8, d_dweight=P, dweight_stride=8)
    for bad in (*bads, dict(d_dloss=None), dict(dx_stride=7), dict(dweight_stride=7)):
        a = _lib.LinearCrossEntropyArgs(**{**good, **bad})
        assert lib.mlkv_linear_cross_entropy_backward(a, None) == _lib.ERR_INVALID, bad
        assert lib.mlkv_linear_cross_entropy_backward_workspace(a) == -1


def _adamw(tensors, **over):
    table = (_lib.AdamWTensor * len(tensors))(*tensors)
    return _lib.AdamWArgs(**{**dict(tensors=table, count=len(tensors), lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1, state_bits=32), **over})


def test_adamw_refusals(lib):
    one = dict(n=8, d_param=P, d_grad=P, d_m=2 * P, d_v=3 * P)
    t = lambda **over: _lib.AdamWTensor(**{**one, **over})  # noqa: E731
    for bad in (dict(n=-1), dict(n=2 ** 40), dict(d_param=None), dict(d_grad=None), dict(d_m=None), dict(d_v=None), dict(param_type=3), dict(grad_type=-1),
                dict(d_copy=P, copy_type=_lib.TYPE_FLOAT), dict(d_copy=P, copy_type=3)):
        assert lib.mlkv_adamw(_adamw([t(**bad)]), None) == _lib.ERR_INVALID, bad
    for bad in (dict(state_bits=16), dict(state_bits=8), dict(count=-1), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=math.nan), dict(eps=-1.0), dict(eps=math.inf),
                dict(weight_decay=math.nan), dict(lr=math.inf), dict(step=0)):
        assert lib.mlkv_adamw(_adamw([t()], **bad), None) == _lib.ERR_INVALID, bad
    # a parameter twice, or a part of it; a state twice; one tensor as both
    apart = dict(d_param=5 * P, d_m=6 * P, d_v=7 * P)
    for other in (dict(d_param=P), dict(d_param=P + 28), dict(d_param=P - 4), dict(d_m=2 * P), dict(d_v=3 * P + 4), dict(d_v=2 * P), dict(d_m=5 * P),
                  dict(d_copy=P, copy_type=_lib.TYPE_BFLOAT)):
        assert lib.mlkv_adamw(_adamw([t(), t(**{**apart, **other})]), None) == _lib.ERR_INVALID, other
    assert lib.mlkv_adamw(_adamw([t(d_v=2 * P)]), None) == _lib.ERR_INVALID
    small = dict(d_scales=8 * P)
    assert lib.mlkv_adamw(_adamw([t(**small), t(**apart, **small)], state_bits=8), None) == _lib.ERR_INVALID
    assert lib.mlkv_adamw(None, None) == _lib.ERR_INVALID


def test_argument_checks_of_the_python_face():
    x, t = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: dense.gated_linear(x, x, x), lambda: dense.linear_cross_entropy(x, x, t), lambda: dense.adamw([x], [x], dense.adamw_state([x]), 1, lr=0.1)):
        with pytest.raises(TypeError, match="CUDA"):
            call()
    with pytest.raises(ValueError):
        dense.adamw_state([x], 4)
    with pytest.raises(ValueError, match="grads"):
        dense.adamw([x], [], dense.adamw_state([x]), 1, lr=0.1)
    with pytest.raises(ValueError, match="state.m"):
        dense.adamw([x], [x], dense.AdamWState([], [], None), 1, lr=0.1)
    with pytest.raises(ValueError, match="seed"):
        dense.adamw([x], [x], dense.adamw_state([x]), 1, lr=0.1, seed=1 << 32)
    state = dense.adamw_state([torch.zeros(3, 100)], 8)
    assert state.m[0].dtype == torch.float8_e4m3fn and state.v[0].shape == (3, 100) and state.scales[0].shape == (2, 2)
    dense.adamw([], [], dense.adamw_state([]), 1, lr=0.1)  # nothing to step


def test_anything_but_cuda_tensors_is_left_to_the_checked_calls(lib):
    from paper_2504_01506_gb300 import _dense_calls as calls

    calls.bind(_lib.LIB_PATH)
    x, t = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    for first in (x, None, 3, [1.0], x[0]):
        assert calls.gated_linear(first, x, x, 3, False) is NotImplemented
        assert calls.gated_linear_backward(x, first, x, x, x, x, 3, True, True) is NotImplemented
        assert calls.linear_cross_entropy(first, x, t, 1.0) is NotImplemented
        assert calls.linear_cross_entropy_backward(t, first, x, t, x, 1.0, True, True) is NotImplemented
        assert calls.adamw([first], [x], [x], [x], None, None, 0.1, 0.9, 0.99, 1e-8, 0.0, 1, None, 0) is NotImplemented
    assert calls.adamw() is NotImplemented
