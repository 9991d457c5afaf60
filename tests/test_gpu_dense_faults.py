"""The products' bounded waits: operands that never come end the kernel with a status, not a hang.

Nothing faults on the device: the kernel's own waits run out (mlkv_debug_fail,
MLKV_FAULT_PRODUCT), it frees what it holds and records MLKV_ERR_TIMEOUT, and the
next product on the same device is right again.
"""
import pytest

from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(300, 520, 200), (4, 4096, 4096), (2, 64, 64), (8192, 2560, 1024)],
                         ids=["single blocks", "a cluster's shares", "one tile", "pairs"])
def test_waits_run_out_and_are_told(m, n, k):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import MLKVError, _lib, dense

    torch.manual_seed(1)
    x, w = torch.randn(m, k, device="cuda").bfloat16(), torch.randn(n, k, device="cuda").bfloat16()
    want = dense.linear(x, w)
    dense.sync()
    lib = _lib.load()
    assert lib.mlkv_debug_fail(_lib.FAULT_PRODUCT, 1) == _lib.OK
    dense.linear(x, w)
    with pytest.raises(MLKVError) as e:
        dense.sync()
    assert e.value.code == _lib.ERR_TIMEOUT
    dense.sync()  # told once
    assert torch.equal(dense.linear(x, w), want)
    dense.sync()


def test_only_the_armed_launch_fails():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import MLKVError, _lib, dense

    x, w = torch.randn(40, 96, device="cuda").half(), torch.randn(72, 96, device="cuda").half()
    lib = _lib.load()
    assert lib.mlkv_debug_fail(_lib.FAULT_PRODUCT, 3) == _lib.OK
    a, b = dense.linear(x, w), dense.linear(x, w)
    dense.sync()
    assert torch.equal(a, b)
    dense.linear(x, w)
    with pytest.raises(MLKVError):
        dense.sync()
    assert lib.mlkv_debug_fail(_lib.FAULT_PRODUCT, 1) == _lib.OK
    assert lib.mlkv_debug_fail(_lib.FAULT_PRODUCT, 0) == _lib.OK  # disarmed
    assert torch.equal(dense.linear(x, w), a)
    dense.sync()
