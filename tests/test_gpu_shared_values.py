"""Attention over shared pages and by sequence at scores that leave a block, a warp's first
one or several heads' without a finite maximum, and at values that the format allows and
random tokens do not reach; against the oracle in fp64."""
import gc

import numpy as np
import pytest
import torch

from tests.gpu_common import require_gpu
from tests.helpers import check_attention, kv_pair
from tests.test_gpu_pages import Shared
from tests.test_gpu_shared import _queries, _reference, _replayed

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


class Edited(Shared):
    """append(n, edit): edit(k, v) changes the new tokens [B, H, L, D] (bf16, on the device)
    before they are appended."""

    def append(self, n, edit=None):
        if edit is None:
            return super().append(n)
        L = max(max(n), 1)
        k, v, _, _ = kv_pair(self.B, self.H, L, self.D, "bf16", seed=self.seed, stream=self.step)
        self.step += 1
        edit(k, v)
        self.gc.append_ragged(k, v, n)
        nk, nv = k.float().cpu().numpy(), v.float().cpu().numpy()
        for b in range(self.B):
            if n[b]:
                new = (nk[b:b + 1, :, :n[b]], nv[b:b + 1, :, :n[b]])
                self.oc[b].append(*new)
                self.hist[b] = tuple(np.concatenate([h, x], 2) for h, x in zip(self.hist[b], new))
        self.n_last = list(n)
        return L


def _decodes(bt, qd):
    return {"shared": bt.gc.attend_decode_shared(qd),
            "shared, captured": _replayed(bt.gc.attend_decode_shared, qd, bt.gc.attend_shared_workspace())}


def _prefills(bt, qd, L):
    return {"shared": bt.gc.attend_prefill_shared(qd),
            "shared, captured": _replayed(bt.gc.attend_prefill_shared, qd, bt.gc.attend_shared_workspace(L))}


def _check(bt, outs, q, rows=None):
    for name, out in outs.items():
        out = out.float().cpu().numpy()
        for b in range(bt.B):
            n = q.shape[2] if rows is None else rows[b]
            if n and bt.oc[b].T:
                with np.errstate(invalid="ignore", over="ignore"):
                    ref = _reference(bt, b, q[b:b + 1, :, :n])
                assert np.isfinite(ref).all()
                check_attention(out[b:b + 1, :, :n], ref, "bf16", f"{name}, sequence {b}")


@pytest.mark.parametrize("H,Hq,D", [(2, 8, 128), (1, 16, 64), (2, 2, 64)])
@pytest.mark.parametrize("shared", [0, 600])
def test_blocks_whose_scores_are_all_minus_infinity(H, Hq, D, shared):
    """Keys of -inf in a channel where the query is 1: tokens without weight, here most of a
    KIVI window, whole blocks of it among them, and the window's first or last block alone."""
    bt = Edited("kivi2", 4, H, Hq, D, 1400, num_pages=30, seed=D + shared)
    if shared:
        bt.append([shared, 0, 0, 0])
        bt.fork([0, 0, 0], [1, 2, 3])

    def edit(k, v):
        k[0, :, 1:, 3] = float("-inf")       # all but one token
        k[1, :, -33:, 3] = float("-inf")     # the last block, and what is before it in part
        k[2, :, :70, 3] = float("-inf")      # the first blocks
        k[3, :, ::2, 3] = float("-inf")
    # (below the window's 128 tokens: an infinite key is never coded)
    L = bt.append([97, 97, 97, 65], edit)
    q = _queries(bt, 1, 3)
    q[..., 3] = 1.0
    _check(bt, _decodes(bt, q.cuda()), q)
    q = _queries(bt, L, 4)
    q[..., 3] = 1.0
    if shared:                               # (without: rows of sequence 2 that see no finite score)
        _check(bt, _prefills(bt, q.cuda(), L), q, bt.n_last)


def test_scores_that_overflow_for_one_head_of_two():
    """Keys of 2^127 in a channel: -inf for a head whose query there is -2^10, finite for its
    neighbour's 2^-120."""
    bt = Edited("kivi2", 3, 1, 4, 64, 900, num_pages=12, seed=8)

    def edit(k, v):
        k[0, :, :64, 5] = 2.0 ** 127
        k[1, :, -40:, 5] = 2.0 ** 127
        k[2, :, 31:64, 5] = 2.0 ** 127
    bt.append([100, 97, 65], edit)
    q = _queries(bt, 1, 5)
    q[:, 0::2, :, 5] = -2.0 ** 10
    q[:, 1::2, :, 5] = 2.0 ** -120
    _check(bt, _decodes(bt, q.cuda()), q)


@pytest.mark.parametrize("fmt", ["kivi2", "kivi4"])
def test_minus_infinity_by_sequence(fmt):
    """The same windows through attend_decode of a cache long enough for its streaming kernel (16
    32-token blocks a SM): each of its warps takes a block in turn, so most begin with such a one."""
    bt = Edited(fmt, 10, 8, 16, 64, 1200, num_pages=60, seed=41)
    bt.append([1000] * 10)

    def edit(k, v):
        k[:, :, :, 3] = float("-inf")
        k[1, :, -1, 3] = 0.5
    bt.append([60] * 10, edit)               # (a kivi4 cache's window keeps 64)
    q = _queries(bt, 1, 3)
    q[..., 3] = 1.0
    out = bt.gc.attend_decode(q.cuda()).float().cpu().numpy()
    for b in (0, 1, 9):
        ref = _reference(bt, b, q[b:b + 1])
        assert np.isfinite(ref).all()
        check_attention(out[b:b + 1], ref, "bf16", f"sequence {b}")


@pytest.mark.parametrize("fmt,H,Hq,D", [("kivi2", 2, 8, 128), ("affine4", 2, 8, 64), ("sym2", 1, 4, 128)])
def test_nan_stays_in_its_row(fmt, H, Hq, D):
    """A NaN query (all of it, or one channel) makes its own row NaN and no other; eagerly and
    captured, prompts short and long enough to go sequence by sequence."""
    bt = Edited(fmt, 4, H, Hq, D, 1600, num_pages=30, seed=2)
    bt.append([600, 0, 0, 0])
    bt.fork([0, 0], [1, 2])
    for n in ([1, 40, 3, 70], [5, 700, 300, 600]):
        L = bt.append(n)
        q = _queries(bt, 1, 6)
        q[0, 1], q[1, 0, 0, 7], q[3, -1] = float("nan"), float("nan"), float("nan")
        bad = np.zeros((bt.B, Hq), bool)
        bad[0, 1] = bad[1, 0] = bad[3, -1] = True
        for name, out in _decodes(bt, q.cuda()).items():
            out = out.float().cpu().numpy()
            for b in range(bt.B):
                assert np.isnan(out[b, bad[b]]).all(), name
                ref = _reference(bt, b, torch.nan_to_num(q[b:b + 1]))
                check_attention(out[b:b + 1, ~bad[b]], ref[:, ~bad[b]], "bf16", name)
        q = _queries(bt, L, 6)
        bad = np.zeros((bt.B, Hq, L), bool)
        for b, h, l in ((0, 1, 0), (1, 0, n[1] - 1), (1, 0, 17), (3, Hq - 1, 64)):
            if l < n[b]:
                q[b, h, l] = float("nan")
                bad[b, h, l] = True
        for name, out in _prefills(bt, q.cuda(), L).items():
            out = out.float().cpu().numpy()
            for b in range(bt.B):
                w, o = bad[b, :, :n[b]], out[b, :, :n[b]]
                assert np.isnan(o[w]).all(), name
                ref = _reference(bt, b, torch.nan_to_num(q[b:b + 1, :, :n[b]]))[0]
                check_attention(o[~w], ref[~w], "bf16", name)


@pytest.mark.parametrize("fmt", ["kivi2", "kivi4"])
@pytest.mark.parametrize("D", [64, 128])
def test_large_offsets(fmt, D):
    """A key channel of +-10,000 to 40,000 with steps of its range, against queries of 2^-13 there:
    offsets of all fp16's range, in the own tokens and in the shared ones."""
    bt = Edited(fmt, 4, 2, 8, D, 1200, num_pages=24, seed=D)

    def edit(k, v):
        k[:, 0, :, 7] = 100 * k[:, 0, :, 7] + 30000
        k[:, 1, :, D - 9] = 100 * k[:, 1, :, D - 9] - 10000
        k[:, 1, :, 2] = 40000
    bt.append([0, 0, 700, 300], edit)
    bt.append([600, 1, 33, 300], edit)
    bt.fork([0], [1])
    L = bt.append([40, 90, 1, 160], edit)
    for n in (1, L):
        q = _queries(bt, n, 9)
        for h, c in ((0, 7), (1, D - 9), (1, 2)):
            q[:, 4 * h:4 * h + 4, :, c] = 2.0 ** -13 * torch.sign(q[:, 4 * h:4 * h + 4, :, c])
        if n == 1:
            _check(bt, _decodes(bt, q.cuda()), q)
        else:
            _check(bt, _prefills(bt, q.cuda(), L), q, bt.n_last)


@pytest.mark.parametrize("fmt,H,Hq,D", [("affine4", 1, 1, 64), ("sym2", 1, 16, 128), ("kivi2", 3, 3, 64),
                                        ("kivi4", 1, 5, 128)])
def test_the_smallest_caches(fmt, H, Hq, D):
    """One sequence (which nothing can be forked into), one token, one page, one row."""
    bt = Edited(fmt, 1, H, Hq, D, 256, num_pages=1, seed=1)
    q = _queries(bt, 1, 2)
    assert all(torch.all(x == 0) for x in _decodes(bt, q.cuda()).values())
    for n in (1, 1, 31, 200, 23):
        L = bt.append([n])
        _check(bt, _decodes(bt, q.cuda()), q)
        p = _queries(bt, L, 3)
        _check(bt, _prefills(bt, p.cuda(), L), p)


def test_a_workspace_of_two_captured_calls():
    """Two caches' graphs over one workspace, replayed in turn on one stream: a call leaves nothing
    in it that a later one reads."""
    a = Edited("kivi2", 6, 2, 8, 128, 1200, num_pages=30, seed=5)
    b = Edited("affine4", 9, 1, 4, 64, 1200, num_pages=40, seed=6)
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    graphs = []
    for bt in (a, b):
        bt.append([700] + [0] * (bt.B - 1))
        bt.fork([0] * (bt.B - 1), list(range(1, bt.B)))
        L = bt.append([1 + i for i in range(bt.B)])
        q, p = _queries(bt, 1, 7), _queries(bt, L, 8)
        qd, pd = q.cuda(), p.cuda()
        for call, x, host, rows in ((bt.gc.attend_decode_shared, qd, q, None), (bt.gc.attend_prefill_shared, pd, p, bt.n_last)):
            out = torch.zeros_like(x)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                call(x, out=out, workspace=ws)
            graphs.append((bt, g, out, host, rows, x))
    for order in ((0, 1, 2, 3), (3, 1, 2, 0), (2, 0, 3, 1)):
        for i in order:
            graphs[i][2].zero_()
            graphs[i][1].replay()
        torch.cuda.synchronize()
        for bt, _, out, host, rows, _ in graphs:
            _check(bt, {"replayed": out}, host, rows)
