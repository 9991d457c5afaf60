"""The extension module of the dense operators' calls, without a GPU: it is built, finds the library, and leaves what it does not take."""
import ctypes
import os
import warnings

import pytest
import torch

from paper_2504_01506_gb300 import _lib, build, dense


@pytest.fixture(scope="module")
def calls():
    build.build()
    from paper_2504_01506_gb300 import _dense_calls

    _dense_calls.bind(_lib.LIB_PATH)
    return _dense_calls


def test_anything_but_cuda_tensors_is_left_to_the_checked_calls(calls):
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    h = x.bfloat16()
    lp = dense.TokenLogprobs(x[:, 0], x[:, 0], x[:, :2], None, None)
    for first in (x, None, 3, [1.0], x[0]):
        assert calls.layer_norm(first, None, None, 1e-5, -1, False) is NotImplemented
        assert calls.layer_norm_backward(first, first, None, x[:, :2], True) is NotImplemented
        assert calls.linear(first, h, None, 0, None, False) is NotImplemented
        assert calls.linear_backward(first, first, h, None, 0, False, True, True) is NotImplemented
        assert calls.token_logprobs(first, t, 0, 1.0) is NotImplemented
        assert calls.token_logprobs_backward(first, t, lp.entropy, lp.stats, None, None, 1.0, False) is NotImplemented
    assert calls.linear() is NotImplemented
    assert dense._native(x) is None and dense._native(None) is None


def test_a_library_without_the_calls_is_refused(calls, tmp_path):
    with pytest.raises(ImportError):
        calls.bind(str(tmp_path / "none.so"))
    calls.bind(_lib.LIB_PATH)


def test_a_status_is_raised():
    with pytest.raises(dense.MLKVError):
        dense._done(_lib.ERR_INVALID)
    assert dense._done((1, 2)) == (1, 2)


def test_without_the_module_the_checked_calls_are_made(calls, monkeypatch):
    """Told once; the library is there all the same."""
    import sys

    import paper_2504_01506_gb300 as package

    class OnGpu:
        is_cuda = True

    monkeypatch.setattr(dense, "_calls", None)
    monkeypatch.delattr(package, "_dense_calls")
    monkeypatch.setitem(sys.modules, "paper_2504_01506_gb300._dense_calls", None)
    with pytest.warns(RuntimeWarning, match="extension module is missing"):
        assert dense._native(OnGpu()) is None
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert dense._native(OnGpu()) is None


@pytest.fixture
def small_build(monkeypatch, tmp_path):
    """A build of one small source, in a folder of its own."""
    (tmp_path / "a.cu").write_text('extern "C" int answer() { return 42; }\n')
    (tmp_path / build.CALLS_SOURCE).write_text("\n")
    monkeypatch.delenv("MLKV_NVCC_FLAGS", raising=False)
    for name, value in dict(CSRC=tmp_path, BUILD=tmp_path / "build", LIB=tmp_path / "lib.so", CALLS=tmp_path / "calls.so").items():
        monkeypatch.setattr(build, name, str(value))
    monkeypatch.setattr(build, "SOURCES", ["a.cu"])
    monkeypatch.setattr(build, "DENSE", [])
    return tmp_path


def test_the_library_is_built_where_the_module_cannot_be(small_build, monkeypatch, capsys):
    """... and an old module, which may be of another library or another torch, does not stay."""
    (small_build / "calls.so").write_text("old")
    def failing(error):
        def build_calls():
            raise error
        return build_calls

    for error in (RuntimeError("no Python.h"), FileNotFoundError("no g++")):
        monkeypatch.setattr(build, "build_calls", failing(error))
        built = build.build()
        assert ctypes.CDLL(built).answer() == 42 and not os.path.exists(build.CALLS)
        assert str(error) in capsys.readouterr().err
    when = os.path.getmtime(built)
    build.build()  # tries the module again, and leaves the library
    assert os.path.getmtime(built) == when


def test_the_module_is_built_anew_with_another_torch(small_build, monkeypatch):
    made = []
    real = build.subprocess.run

    def run(cmd, **kw):
        if build.CALLS_SOURCE in " ".join(cmd):
            made.append(cmd)
            cmd = ["cp", os.path.join(build.CSRC, build.CALLS_SOURCE), cmd[cmd.index("-o") + 1]]
        return real(cmd, **kw)

    monkeypatch.setattr(build.subprocess, "run", run)
    build.build()
    build.build()
    assert len(made) == 1 and build.up_to_date()
    monkeypatch.setattr(build, "_torch_version", lambda: "0.0")
    assert not build.up_to_date()
    build.build()
    assert len(made) == 2 and build.up_to_date()
