"""The extension module of the dense operators' calls, without a GPU: it is built, finds the library, and leaves what it does not take."""
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
