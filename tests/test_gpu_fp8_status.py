"""zc_fp8_status with several streams and threads."""
import threading

import pytest
import torch

from paper_2508_19263_b200 import binding as zc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_no_report_is_lost_between_queries():
    """One thread asks for the status again and again on a stream of its own, another makes products whose waits run out, one at a time.
    When a product is done and the status has been asked for once more, one of the two has to have heard of it."""
    q = lambda r: zc.fp8_quantize(torch.ones((r, 256), device=DEV), zc.fp8_empty(r, 256))  # noqa: E731
    a, b, d = q(64), q(128), torch.empty((64, 128), device=DEV)
    torch.cuda.synchronize()
    heard, stop, lock, failures = 0, False, threading.Lock(), []

    def ask(stream):
        nonlocal heard
        status = zc.fp8_status(stream)
        if status == zc.E_DEVICE_TIMEOUT:
            with lock:
                heard += 1
        elif status != zc.OK:
            failures.append(status)

    def poll():
        stream = torch.cuda.Stream()
        while not stop:
            ask(stream)

    assert zc.fp8_status() == zc.OK
    own, asking, lost = torch.cuda.Stream(), torch.cuda.Stream(), 0
    poller = threading.Thread(target=poll)
    try:
        zc.test_set_wait_limit(20)
        zc.test_stall_decoder(True)                                          # no copies are started
        poller.start()
        for _ in range(400):
            with lock:
                before = heard
            zc.fp8_matmul(a, b, d, stream=own)
            own.synchronize()
            ask(asking)
            # a query of the other thread may have taken the mark and not have counted it yet
            for _ in range(2000):
                with lock:
                    if heard > before:
                        break
                threading.Event().wait(0.0005)
            else:
                lost += 1
                if lost == 3:
                    break
    finally:
        zc.test_set_wait_limit(0)
        zc.test_stall_decoder(False)
        stop = True
        poller.join()
    assert not failures and lost == 0
    assert zc.fp8_status() == zc.OK
    zc.fp8_matmul(a, b, d)
    assert bool((d == 256).all()) and zc.fp8_status() == zc.OK


def test_a_capture_goes_on():
    x = torch.ones((64, 256), device=DEV)
    a, b, d = zc.fp8_empty(64, 256), zc.fp8_quantize(torch.ones((128, 256), device=DEV), zc.fp8_empty(128, 256)), torch.zeros((64, 128), device=DEV)
    zc.fp8_quantize(x, a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        zc.fp8_quantize(x, a)
        assert zc.fp8_status() == zc.E_CUDA                                  # on the stream that is captured
        zc.fp8_matmul(a, b, d)
    x.fill_(2.0)
    g.replay()
    torch.cuda.synchronize()
    assert bool((d == 512).all()) and zc.fp8_status() == zc.OK
