"""The products' bounded waits: operands that never come end the kernel with a status, not a hang.

Nothing faults on the device: the kernel's own waits run out (mlkv_debug_fail,
MLKV_FAULT_PRODUCT), it frees what it holds and records MLKV_ERR_TIMEOUT, and the
next product on the same device is right again.
"""
import threading
import time

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


def test_told_to_whoever_asks_and_not_lost():
    """A wait that runs out on one stream while others ask again and again: told at least once, and not any more after that."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import MLKVError, _lib, dense

    torch.manual_seed(2)
    x, w = torch.randn(300, 200, device="cuda").bfloat16(), torch.randn(520, 200, device="cuda").bfloat16()
    want = dense.linear(x, w)
    dense.sync()
    lib = _lib.load()
    told, stop = [], threading.Event()

    def ask():
        with torch.cuda.stream(torch.cuda.Stream()):
            while not stop.is_set():
                try:
                    dense.sync()
                except MLKVError as e:
                    told.append(e.code)

    threads = [threading.Thread(target=ask) for _ in range(3)]
    for t in threads:
        t.start()
    for n in range(2):
        before = len(told)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            assert lib.mlkv_debug_fail(_lib.FAULT_PRODUCT, 1) == _lib.OK
            dense.linear(x, w)
            side.synchronize()
            try:
                dense.sync()
            except MLKVError as e:
                told.append(e.code)
        until = time.monotonic() + 10  # (a thread that has been told may not have noted it yet)
        while len(told) == before and time.monotonic() < until:
            time.sleep(0.001)
        assert len(told) > before
    stop.set()
    for t in threads:
        t.join()
    assert set(told) == {_lib.ERR_TIMEOUT}
    dense.sync()
    assert torch.equal(dense.linear(x, w), want)
    dense.sync()
