"""Captured calls on ragged and paged caches: what is refused, what a replay may do to a cache that
has been forked, cut and compacted since, and what the host finds after kvq_cache_sync."""
import numpy as np
import pytest
import torch

from paper_2609_04263_gb300 import kvq
from tests.gpu_common import require_gpu
from tests.test_gpu_pages import PAGED, RAGGED, Shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _refused_in_capture(call, status=kvq.KVQ_ERR_UNSUPPORTED):
    torch.cuda.synchronize()
    graph, keep = torch.cuda.CUDAGraph(), torch.zeros(1, device="cuda")
    with torch.cuda.graph(graph):
        keep += 1
        with pytest.raises(kvq.KvqError) as ei:
            call()
    assert ei.value.status == status


def test_a_release_before_forks_is_not_captured():
    """Replayed behind a fork of the sequence it would empty, it would leave it without tokens but
    with pages that the fork shares, and the next append would write into those."""
    bt = Shared("affine4", 3, 1, 4, 64, 800, num_pages=9, seed=3)
    bt.append([10, 600, 0])
    _refused_in_capture(lambda: bt.gc.seq_release(1))
    assert bt.gc.free_pages() == 9 - 4
    bt.fork([1], [2])
    bt.gc.sync()
    L = bt.append([1, 5, 3])
    bt.check(L)


def test_a_ragged_release_is_captured():
    bt = Shared("affine4", 2, 1, 4, 64, 512, layout=RAGGED, seed=4)
    bt.append([20, 30])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        bt.gc.seq_release(1)
    graph.replay()
    bt.gc.sync()
    bt.set(1, bt.hist[1], 0)
    bt.check()
    bt.append([1, 40])
    graph.replay()
    bt.gc.sync()
    bt.set(1, bt.hist[1], 0)
    bt.check()
