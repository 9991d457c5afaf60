"""The dense operators' binding against their header, and their refusals, without a GPU."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2504_01506_gb300 import _lib, build, dense

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "mlkv_dense.h")


def _source():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def test_every_declared_call_is_bound_with_its_arguments(lib):
    arity = {}
    for m in re.finditer(r"\b(mlkv_[a-z_]+)\s*\(([^)]*)\)\s*;", _source(), flags=re.S):
        arity[m.group(1)] = " ".join(m.group(2).split()).count(",") + 1
    assert sorted(arity) == sorted(_lib.EXPORTED_DENSE)
    for name, n in arity.items():
        assert len(getattr(lib, name).argtypes) == n, name


def test_constants_match_the_header():
    defines = {m.group(1): int(m.group(2)) for m in re.finditer(r"#define MLKV_(\w+) (\d+)\b", _source())}
    assert {"TYPE_FLOAT", "TYPE_BFLOAT", "TYPE_HALF", "ACT_NONE", "ACT_RELU", "ACT_GELU_TANH", "ACT_SILU", "MAX_TOP"} <= set(defines)
    for name, value in defines.items():
        assert getattr(_lib, name) == value, name


def test_argument_struct_matches_the_header(tmp_path):
    fields = [f for f, _ in _lib.LinearArgs._fields_]
    prog = tmp_path / "layout.c"
    body = "".join(f'printf("{f} %zu\\n", offsetof(mlkv_linear_args, {f}));' for f in fields)
    prog.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mlkv_dense.h"\n'
                    f'int main(void){{printf("size %zu\\n", sizeof(mlkv_linear_args));{body}return 0;}}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.dirname(HEADER), str(prog), "-o", str(exe)], check=True)
    out = dict(ln.split() for ln in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(out["size"]) == ctypes.sizeof(_lib.LinearArgs)
    for f in fields:
        assert int(out[f]) == getattr(_lib.LinearArgs, f).offset, f


P = 4096  # a pointer that no call here reads


def test_layer_norm_refusals(lib):
    good = dict(x=P, xs=8, xt=0, rows=4, dim=8, w=P, b=P, wt=0, eps=1e-5, y=P, ys=8, yt=1, stats=None, stream=None)
    for bad in (dict(x=None), dict(xs=7), dict(xt=3), dict(xt=-1), dict(rows=-1), dict(rows=2 ** 31), dict(dim=0), dict(dim=2 ** 20),
                dict(wt=9), dict(eps=-1.0), dict(eps=float("nan")), dict(y=None), dict(ys=7), dict(yt=3), dict(xt=1, yt=2),
                dict(xt=2, yt=0)):
        assert lib.mlkv_layer_norm(*{**good, **bad}.values()) == _lib.ERR_INVALID, bad
    good = dict(dy=P, dys=8, dyt=1, x=P, xs=8, xt=0, rows=4, dim=8, w=P, wt=0, stats=P, dx=P, dxs=8, dw=P, db=P, ws=P, wsb=1 << 30,
                stream=None)
    for bad in (dict(dy=None), dict(dys=7), dict(dyt=4), dict(x=None), dict(xs=1), dict(rows=-1), dict(dim=0), dict(wt=-2),
                dict(stats=None), dict(dxs=7)):
        assert lib.mlkv_layer_norm_backward(*{**good, **bad}.values()) == _lib.ERR_INVALID, bad
    assert lib.mlkv_layer_norm_backward_workspace(-1, 8) == -1
    assert lib.mlkv_layer_norm_backward_workspace(4, 0) == -1


def test_logprobs_refusals(lib):
    good = dict(x=P, s=8, t=0, n=2, v=8, tg=P, scale=1.0, top=2, lp=P, e=P, st=P, tl=P, ti=P, ws=None, wsb=0, stream=None)
    for bad in (dict(x=None), dict(s=7), dict(t=5), dict(n=-1), dict(n=2 ** 31), dict(v=0), dict(v=2 ** 30), dict(tg=None), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(top=-1), dict(top=33), dict(lp=None),
                dict(e=None), dict(st=None), dict(tl=None), dict(ti=None)):
        assert lib.mlkv_token_logprobs(*{**good, **bad}.values()) == _lib.ERR_INVALID, bad
    good = dict(x=P, s=8, t=0, n=2, v=8, tg=P, scale=1.0, e=P, st=P, g=P, h=P, dz=P, dzs=8, stream=None)
    for bad in (dict(x=None), dict(s=7), dict(t=5), dict(n=-1), dict(v=0), dict(tg=None), dict(scale=0.0), dict(st=None),
                dict(e=None), dict(dz=None), dict(dzs=7), dict(dzs=9)):
        assert lib.mlkv_token_logprobs_backward(*{**good, **bad}.values()) == _lib.ERR_INVALID, bad


def test_linear_refusals(lib):
    good = dict(m=4, n=8, k=8, d_x=P, x_stride=8, d_weight=P, weight_stride=8, d_y=P, y_stride=8, type=_lib.TYPE_BFLOAT,
                activation=_lib.ACT_SILU)
    bads = (dict(m=-1), dict(n=-1), dict(k=-1), dict(m=2 ** 31), dict(type=_lib.TYPE_FLOAT), dict(type=7), dict(activation=4),
            dict(activation=-1), dict(d_x=None), dict(x_stride=7), dict(d_weight=None), dict(weight_stride=7), dict(x_stride=2 ** 38))
    for bad in (*bads, dict(d_y=None), dict(y_stride=7), dict(d_pre=P, pre_stride=7), dict(d_residual=P, residual_stride=1)):
        a = _lib.LinearArgs(**{**good, **bad})
        assert lib.mlkv_linear(a, None) == _lib.ERR_INVALID, bad
        assert lib.mlkv_linear_workspace(a) == -1
    good.update(d_dy=P, dy_stride=8, d_pre=P, pre_stride=8, d_dx=P, dx_stride=8, d_dweight=P, dweight_stride=8)
    for bad in (*bads, dict(d_dy=None), dict(dy_stride=7), dict(d_pre=None), dict(pre_stride=2), dict(dx_stride=7), dict(dweight_stride=7)):
        a = _lib.LinearArgs(**{**good, **bad})
        assert lib.mlkv_linear_backward(a, None) == _lib.ERR_INVALID, bad
        assert lib.mlkv_linear_backward_workspace(a) == -1
    assert lib.mlkv_linear(None, None) == _lib.ERR_INVALID


def test_matrices_with_rows_that_are_not_contiguous_are_copied():
    x = torch.randn(6, 8)
    assert dense._matrix(x, "x") is x
    assert dense._matrix(x[:, 2:5], "x").data_ptr() == x[:, 2:5].data_ptr()
    for y in (x.t(), x[:1].expand(4, 8), x[:, ::2]):
        z = dense._matrix(y, "x")
        assert z.is_contiguous() and torch.equal(z, y)
    assert dense._row_stride(x[:, 2:5]) == 8 and dense._row_stride(x[:1]) == 8 and dense._row_stride(x[:0]) == 8


def test_argument_checks_of_the_python_face():
    x = torch.zeros(4, 8)
    for call in (lambda: dense.layer_norm(x), lambda: dense.linear(x.bfloat16(), x.bfloat16()),
                 lambda: dense.token_logprobs(x, torch.zeros(4, dtype=torch.int64))):
        with pytest.raises(TypeError, match="CUDA"):
            call()
    with pytest.raises(TypeError):
        dense._matrix(x.double(), "x")
    with pytest.raises(TypeError):
        dense._matrix(x[0], "x")
    with pytest.raises(TypeError):
        dense._matrix([1.0], "x")
    with pytest.raises(TypeError):
        dense._matrix(x, "x", (torch.bfloat16,))
    with pytest.raises(ValueError):
        dense._matrix(x, "x", None, (4, 7))
    with pytest.raises(TypeError):
        dense._matrix(x, "x", None, None, torch.device("cuda", 0))
    with pytest.raises(TypeError):
        dense._vector(torch.zeros(8, dtype=torch.int32), "targets", 8, x.device, (torch.int64,))
    with pytest.raises(ValueError):
        dense._vector(torch.zeros(7), "bias", 8, x.device, (torch.float32,))
    with pytest.raises(ValueError):
        dense._matrix(x, "x", None, (1, 8))
    with pytest.raises(dense.MLKVError):
        dense._workspace(-1, x.device)


def test_sync_of_a_device_without_an_index_is_the_current_ones(monkeypatch):
    asked = []
    monkeypatch.setattr(dense, "_current_device", lambda: 3)
    monkeypatch.setattr(dense.torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(dense, "_stream", lambda device: None)
    monkeypatch.setattr(dense, "_call", lambda device, call, *args: asked.append(device))
    for device in (None, "cuda", torch.device("cuda"), "cuda:1", torch.device("cuda", 2), 0):
        dense.sync(device)
    assert asked == [torch.device("cuda", i) for i in (3, 3, 3, 1, 2, 0)]
    with pytest.raises(TypeError, match="CUDA"):
        dense.sync("cpu")
