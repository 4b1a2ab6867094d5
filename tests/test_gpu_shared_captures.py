"""Captured calls on ragged and paged caches: what is refused, what a replay may do to a cache that
has been forked, cut and compacted since, and what the host finds after kvq_cache_sync."""
import gc

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


@pytest.fixture(autouse=True)
def _no_graph_left():
    """A graph that a caught exception's frames still hold is freed here: freed in the middle of
    another capture, it would end that one."""
    gc.collect()
    yield
    gc.collect()


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


class Replayed(Shared):
    """record(n): an append of n captured; replay(ok): replayed, and followed by the oracle where
    it has to be taken."""

    def record(self, n):
        from tests.helpers import kv_pair
        self.k, self.v, nk, nv = kv_pair(self.B, self.H, max(n), self.D, "bf16", seed=self.seed, stream=99)
        self.n, self.new = n, (nk, nv)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.gc.append_ragged(self.k, self.v, n)
        self.gc.sync()                        # (the host counted the capture)

    def replay(self, times, ok=True):
        for _ in range(times):
            self.graph.replay()
        torch.cuda.synchronize()
        if not ok:
            with pytest.raises(kvq.KvqError) as ei:
                self.gc.sync()
            assert ei.value.status == kvq.KVQ_ERR_CAPACITY
        self.gc.sync()
        for _ in range(times if ok else 0):
            for b in range(self.B):
                if self.n[b]:
                    x = tuple(a[b:b + 1, :, :self.n[b]] for a in self.new)
                    self.oc[b].append(*x)
                    self.hist[b] = tuple(np.concatenate([h, y], 2) for h, y in zip(self.hist[b], x))
        self.n_last = list(self.n) if ok else [0] * self.B


@pytest.mark.parametrize("fmt", ["affine4", "kivi2"])
def test_a_replayed_append_keeps_to_its_pages(fmt):
    """Behind the last page of a sequence stand stale entries of the page table: of a roll-back, of
    the longer sequence that a fork replaced, of pages that compaction has moved.  Their pages
    are others' by then."""
    bt = Replayed(fmt, 4, 2, 8, 64 if fmt == "affine4" else 128, 1536, num_pages=18, seed=11)
    cut = 250 if fmt == "affine4" else 0      # (KIVI cuts to nothing, then starts again)
    bt.append([900, 0, 0, 100])
    bt.record([2, 0, 0, 1])
    bt.replay(3)
    bt.check(2)
    bt.truncate([0], [cut])
    if cut == 0:
        bt.append([250, 0, 0, 0])
    bt.append([0, 800, 300, 0])               # takes the pages that sequence 0 gave up
    bt.replay(3)                              # 256 tokens of sequence 0
    bt.check(2)
    for _ in range(2):
        bt.replay(1, ok=False)
        bt.check(2)
    bt.fork([2], [3])                         # where a replay would still fit
    bt.gc.compact()
    bt.replay(1, ok=False)                    # (sequence 0 holds it up)
    bt.check(2)
    bt.append([1, 0, 0, 0])                   # an eager append takes the page
    bt.replay(5)
    bt.check(2)
    bt.fork([1], [0])
    bt.replay(4)
    bt.check(2)


def test_a_captured_append_takes_no_page():
    bt = Shared("affine4", 2, 1, 4, 64, 1024, num_pages=6, seed=12)
    bt.append([256, 200])
    k = torch.zeros(2, 1, 60, 64, dtype=torch.bfloat16, device="cuda")
    _refused_in_capture(lambda: bt.gc.append_ragged(k, k, [1, 1]))
    _refused_in_capture(lambda: bt.gc.append_ragged(k, k, [0, 57]))
    assert bt.gc.free_pages() == 4
    L = bt.append([3, 60])
    bt.check(L)


@pytest.mark.parametrize("layout", [PAGED, RAGGED])
def test_a_replayed_append_keeps_to_max_tokens(layout):
    """max_tokens inside a page and inside a 64-token chunk."""
    bt = Replayed("sym2", 3, 2, 4, 128, 301, layout=layout, num_pages=7 if layout == PAGED else 0, seed=13)
    bt.append([290, 280, 20])
    bt.record([3, 1, 0])
    bt.replay(3)
    bt.check(3)
    bt.replay(1, ok=False)
    bt.check(3)
    bt.truncate([0], [270])
    bt.replay(4)
    bt.check(3)


def test_an_eager_append_without_the_sync_of_replays_is_refused():
    """The host counts fewer tokens than replays have left, and takes too few pages."""
    bt = Replayed("affine2", 2, 2, 4, 64, 1024, num_pages=8, seed=14)
    bt.append([500, 300])
    bt.record([4, 4])
    for _ in range(2):
        bt.graph.replay()
    k = torch.zeros(2, 2, 10, 64, dtype=torch.bfloat16, device="cuda")
    bt.gc.append_ragged(k, k, [10, 10])       # 500 + 10 for the host, 508 + 10 in truth
    with pytest.raises(kvq.KvqError) as ei:
        bt.gc.sync()
    assert ei.value.status == kvq.KVQ_ERR_CAPACITY
    assert [bt.gc.seq_tokens(b) for b in range(2)] == [508, 308]
    for _ in range(2):
        for b in range(2):
            x = tuple(a[b:b + 1] for a in bt.new)
            bt.oc[b].append(*x)
            bt.hist[b] = tuple(np.concatenate([h, y], 2) for h, y in zip(bt.hist[b], x))
    bt.n_last = [0, 0]
    bt.check()
    L = bt.append([10, 10])
    bt.check(L)


def test_the_first_call_is_not_captured():
    """It zeroes the cache's state, and a replay would do so again behind later appends."""
    bt = Shared("affine4", 2, 1, 4, 64, 512, num_pages=4, seed=15)
    q = torch.randn(2, 4, 1, 64, device="cuda").bfloat16()
    k = q[:, :1].contiguous()
    out, ws = torch.zeros_like(q), torch.empty(bt.gc.attend_shared_workspace(), dtype=torch.uint8, device="cuda")
    calls = (lambda: bt.gc.attend_decode_shared(q, out=out, workspace=ws),
             lambda: bt.gc.attend_prefill_shared(q, out=out, workspace=ws),
             lambda: bt.gc.attend_decode(q, out=out), lambda: bt.gc.append_ragged(k, k, [0, 0]))
    for call in calls:
        _refused_in_capture(call)
    bt.append([300, 2])
    bt.check(300)
    bt.gc.reset()
    for call in calls:
        _refused_in_capture(call)
    for b in range(2):
        bt.set(b, bt.hist[b], 0)
    bt.append([3, 290])
    bt.check(290)
