"""Adapters, group norm and gradient clipping where threads share an object or tensors share memory, on the device."""
import threading

import pytest
import torch

from paper_2407_12637_b200 import cnn

pytestmark = pytest.mark.gpu


def test_two_threads_share_a_group_norm():
    """Images too large for a cluster, two launches a pass, on the default stream: the bits that each thread gets alone."""
    norm = cnn.GroupNorm(24, 3, act="silu")
    xs = [torch.randn(2, 40000, 24, device="cuda") * (i + 1) + i for i in range(2)]
    want, got = [norm.forward(x) for x in xs], [[], []]

    def work(i):
        for _ in range(100):
            got[i].append(norm.forward(xs[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(2) for y in got[i])
