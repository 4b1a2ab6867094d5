"""Trees of more runs than are attended as such, and captured calls behind changes of the tree:
outputs relative to their own size, so that a page left out or attended twice is seen in
sequences of tens of thousands of tokens too.

The bound is 0.0024 of a row's norm: the result's rounding to bf16 is uniform within 2^-8 of a
value at most, 2^-8 / sqrt(3) = 0.00226 root mean square, and P and the values in fp16
(2^-11 each, of terms that average) add below 0.0005.  That a page more or less lies outside of
it, whatever the rounding (more than twice the bound away), is checked on the reference itself,
page by page."""
import gc

import numpy as np
import pytest
import torch

from oracle import kvq_oracle as O
from tests.gpu_common import require_gpu
from tests.test_gpu_pages import PG, Shared
from tests.test_gpu_shared import _captured, _queries

pytestmark = pytest.mark.gpu
BOUND = 0.0024


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


def _by_page(oc, q):
    """Attention of queries [1, Hq, 1, D] over a sequence, its sums kept by page of tokens:
    softmax sums [Hq, pages] and weighted values [Hq, pages, D], of one common maximum."""
    k, v = (np.asarray(x, np.float64)[0] for x in oc.reconstruct())      # [H, T, D]
    qq = np.asarray(q.double().numpy())[0, :, 0]
    rep = qq.shape[0] // k.shape[0]
    Z, N = [], []
    for h in range(qq.shape[0]):
        s = k[h // rep] @ qq[h] / np.sqrt(qq.shape[1])
        p = np.exp(s - s.max())
        cut = range(0, len(p), PG)
        Z.append([p[i:i + PG].sum() for i in cut])
        N.append([p[i:i + PG] @ v[h // rep][i:i + PG] for i in cut])
    return np.array(Z), np.array(N)


def _off(a, ref):
    return np.linalg.norm(a - ref) / np.linalg.norm(ref)


def check_close(bt, b, outs, q, pages=True):
    """Each out [B, Hq, 1, D] of sequence b within BOUND; with pages, a page left out or attended
    twice would not be."""
    Z, N = _by_page(bt.oc[b], q[b:b + 1])
    z, n = Z.sum(1)[:, None], N.sum(1)
    ref = n / z
    np.testing.assert_allclose(ref, O.attend(bt.oc[b], q[b:b + 1].float().numpy())[0, :, 0], rtol=1e-6,
                               atol=1e-9)
    for out in outs:
        err = _off(out[b, :, 0].double().cpu().numpy(), ref)
        assert err <= BOUND, (b, err)
    for i in range(Z.shape[1]) if pages and Z.shape[1] > 1 else ():
        if i == Z.shape[1] - 1 and bt.oc[b].T % PG and bt.oc[b].T % PG < PG // 2:
            continue                              # (a last page of a few tokens)
        for sign in (-1, 1):
            wrong = (n + sign * N[:, i]) / (z + sign * Z[:, i:i + 1])
            assert _off(wrong, ref) > 2 * BOUND, (b, i, sign)


def _both(bt, q):
    qd = q.cuda()
    graph, out = _captured(bt.gc.attend_decode_shared, qd, bt.gc.attend_shared_workspace())
    graph.replay()
    torch.cuda.synchronize()
    return [bt.gc.attend_decode_shared(qd), out]


def test_a_chain_of_more_runs_than_the_plan_holds():
    """Each sequence forks the one before and is a page longer: 79 runs, of which 64 are
    attended as such."""
    B = 80
    bt = Shared("sym2", B, 1, 2, 64, PG * B + 64, num_pages=3 * B + 20, seed=9)
    bt.append([PG] + [0] * (B - 1))
    for b in range(1, B):
        bt.gc.fork([b - 1], [b])
        bt.set(b, bt.hist[b - 1], bt.oc[b - 1].T)
        n = [0] * B
        n[b] = PG if b < B - 1 else 7
        bt.append(n)
    q = _queries(bt, 1, 7)
    outs = _both(bt, q)
    for b in (0, 1, 5, 40, 62, 63, 64, 65, 66, 78, 79):
        check_close(bt, b, outs, q)
    bt.append([1] * B)
    outs = _both(bt, q) + [bt.gc.attend_prefill_shared(q.cuda())]
    for b in (0, 40, 64, 66, 79):
        check_close(bt, b, outs, q)


@pytest.mark.parametrize("fmt", ["affine4", "sym2"])
def test_pairs_of_more_runs_than_the_plan_holds(fmt):
    """A page that all share, then 70 pairs that share one to three more each: the runs kept are
    those that save most, the others' pages are their two members' own."""
    pairs = 70
    B = 2 * pairs
    bt = Shared(fmt, B, 1, 2, 64, 1600, num_pages=1 + 5 * B, seed=21)
    first = list(range(0, B, 2))
    bt.append([PG] + [0] * (B - 1))
    bt.fork([0] * (pairs - 1), first[1:])
    bt.append([PG * (1 + b // 2 % 3) + 3 if b % 2 == 0 else 0 for b in range(B)])
    bt.fork(first, [b + 1 for b in first])
    bt.append([1 + b % 5 for b in range(B)])
    q = _queries(bt, 1, 7)
    outs = _both(bt, q)
    for b in list(range(0, 14)) + [63, 64, 127, 128, 138, 139]:
        check_close(bt, b, outs, q)


def test_captured_calls_follow_later_trees():
    """They follow forks, roll-backs and appends.  The room that the call asks for without forks (a
    unit a sequence and kv head, which a prefill's own tokens may need) does for a decode of fewer
    runs than that."""
    bt = Shared("affine4", 6, 2, 8, 64, 1200, num_pages=40, seed=1)
    bt.append([600, 40, 0, 0, 0, 0])
    q = _queries(bt, 1, 7)
    qd = q.cuda()
    room = bt.gc.attend_shared_workspace()
    bt.gc.attend_decode_shared(qd)
    graphs = [_captured(bt.gc.attend_decode_shared, qd, n) for n in (room + 64 * 256 * 66 * 4, room)]

    def follow():
        assert bt.gc.attend_shared_workspace() > room
        for graph, out in graphs:
            out.fill_(5)
            graph.replay()
            torch.cuda.synchronize()
            bt.gc.sync()
            for b in range(bt.B):
                if bt.oc[b].T:
                    check_close(bt, b, [out], q, pages=False)
                else:
                    assert torch.all(out[b] == 0)

    bt.fork([0, 0, 0], [2, 3, 4])
    follow()
    bt.append([1, 2, 3, 4, 300, 0])
    follow()
    bt.truncate([1], [0])
    follow()
    bt.fork([2, 3], [1, 5])
    bt.append([0, 1, 0, 0, 0, 1])
    follow()
    bt.truncate([4], [513])
    bt.release(0)
    bt.gc.compact()
    follow()
