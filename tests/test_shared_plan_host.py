"""The host's side of shared pages over a CUDA runtime that launches nothing (no GPU): what reaches
the device's plan of shared runs when a launch fails on the way."""
import ctypes
import glob
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
B, PAGE, HEAD, NODE = 5, 256, 8, 8            # (the plan's words: a head, 64 nodes of 8, 3 a sequence)
WORDS = HEAD + 64 * NODE + 3 * B


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    from paper_2609_04263_gb300 import build, kvq
    build.build()
    objects = sorted(glob.glob(os.path.join(build.OUT_DIR, "*.o")))
    if not shutil.which("g++") or not objects:
        pytest.skip("no g++ or no objects")
    so = str(tmp_path_factory.mktemp("fake") / "libkvq_fake.so")
    subprocess.run(["g++", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-o", so, *objects,
                    os.path.join(ROOT, "tests", "fake_cuda_runtime.cpp")], check=True)
    fake = ctypes.CDLL(so)
    for name, (res, args) in kvq._SIGS.items():
        getattr(fake, name).restype, getattr(fake, name).argtypes = res, args
    fake.fake_plan.restype = ctypes.POINTER(ctypes.c_int32)
    fake.fake_fail.argtypes = [ctypes.c_char_p, ctypes.c_int]
    return fake


class Host:
    """A paged cache on the fake runtime."""

    def __init__(self, lib):
        from paper_2609_04263_gb300 import kvq
        self.lib, self.kvq = lib, kvq
        d = kvq.kvq_cache_desc(fmt=kvq.KVQ_FMT_AFFINE, key_bits=4, value_bits=4, group_size=32,
                               residual_tokens=0, sink_tokens=0, norm_iters=8, batch=B, kv_heads=2,
                               q_heads=8, head_dim=64, max_tokens=4096, dtype=kvq.KVQ_BF16,
                               layout=kvq.KVQ_LAYOUT_PAGED, num_pages=60)
        self.h = ctypes.c_void_p()
        assert lib.kvq_create_cache(ctypes.byref(d), 1 << 32, lib.kvq_cache_bytes(ctypes.byref(d)),
                                    ctypes.byref(self.h)) == 0

    def call(self, name, *args):
        a = [(ctypes.c_int * len(x))(*x) if isinstance(x, list) else x for x in args]
        return getattr(self.lib, name)(self.h, *a, None)

    def append(self, n):
        return self.call("kvq_append_pack_ragged", 1 << 33, 1 << 34, max(n), n)

    def fork(self, src, dst):
        return self.call("kvq_seq_fork", len(src), src, dst, None)

    def decode(self):
        n = self.lib.kvq_attend_shared_workspace(self.h, 1)
        return self.call("kvq_attend_decode_shared", 1 << 35, 8, 0.1, 1 << 36, 1 << 37, n)

    def plan(self):
        return np.ctypeslib.as_array(self.lib.fake_plan(), (WORDS,)).copy()


def _steps(x):
    """Calls that change the tree of shared runs."""
    return [lambda: x.append([1000, 0, 0, 0, 20]),
            lambda: x.fork([0, 0], [1, 2]),
            lambda: x.append([300, 600, 0, 0, 1]),
            lambda: x.fork([1], [3]),
            lambda: x.call("kvq_seq_truncate", 1, [2], [300]),
            lambda: x.call("kvq_seq_release", 0),
            lambda: x.fork([3, 1], [0, 4])]


def _nodes(plan):
    return [tuple(plan[HEAD + NODE * i:HEAD + NODE * i + 5]) for i in range(plan[0])]


def _plans(lib):
    x, out = Host(lib), []
    for step in _steps(x):
        assert step() == 0
        out.append(x.plan())
    return out


def test_the_plan_of_a_tree(lib):
    plans = _plans(lib)
    # (first and last page, members, parent): three of 3 pages; then two of 6 under them
    assert [(n[0], n[1], n[3], n[4]) for n in _nodes(plans[1])] == [(0, 3, 3, 0)]
    assert [(n[0], n[1], n[3], n[4]) for n in _nodes(plans[3])] == [(0, 3, 4, 0), (3, 6, 2, 1)]


@pytest.mark.parametrize("k", [1, 3, 4, 5, 6])
@pytest.mark.parametrize("part", [b"plan_words", b"take_kernel", b"change_kernel", b"seq_reset"])
def test_a_failed_launch_leaves_no_stale_plan(lib, part, k):
    """The call says so; whatever comes next sends the whole plan, be it a call on sequences or an
    attention call."""
    from paper_2609_04263_gb300 import kvq
    plans = _plans(lib)
    for attend in (False, True):
        x, failed = Host(lib), False
        for i, step in enumerate(_steps(x)):
            if i == k:
                lib.fake_fail(part, 0)
            st = step()
            if st != 0:
                assert i == k and st == kvq.KVQ_ERR_CUDA
                failed = True
                if part == b"seq_reset":      # nothing was released
                    assert step() == 0
                    failed = False
            lib.fake_fail(b"", -1)
            if failed and not attend:
                continue
            if failed:
                assert x.decode() == 0
                failed = False
            np.testing.assert_array_equal(x.plan(), plans[i])
            if i > k:
                break
        assert x.decode() == 0
        np.testing.assert_array_equal(x.plan(), plans[i])
        lib.kvq_destroy_cache(x.h)


def test_an_attention_call_says_so_when_the_plan_cannot_be_sent(lib):
    from paper_2609_04263_gb300 import kvq
    x = Host(lib)
    steps = _steps(x)
    assert steps[0]() == 0
    lib.fake_fail(b"plan_words", 0)
    assert steps[1]() == kvq.KVQ_ERR_CUDA
    lib.fake_fail(b"plan_words", 0)
    assert x.decode() == kvq.KVQ_ERR_CUDA
    n = lib.fake_launches()
    lib.fake_fail(b"", -1)
    assert x.decode() == 0 and lib.fake_launches() == n + 4     # the words, then the three kernels
    assert x.decode() == 0 and lib.fake_launches() == n + 7
    lib.kvq_destroy_cache(x.h)


def test_no_host_memory(lib):
    """Each allocation of each call fails in turn: the call says so (or, where the tree of shared runs
    alone had no room, goes on without one), nothing is half done, and made again it succeeds."""
    from paper_2609_04263_gb300 import kvq
    plans = _plans(lib)

    def pages(h):
        return (lib.kvq_free_pages(h), [lib.kvq_seq_tokens(h, b) for b in range(B)],
                [lib.kvq_seq_pages(h, b, None, 0) for b in range(B)])
    for i, plan in enumerate(plans):
        for k in range(200):
            x = Host(lib)
            for before in _steps(x)[:i]:
                assert before() == 0
            was = pages(x.h)
            lib.fake_no_memory(k)
            st = _steps(x)[i]()
            reached = lib.fake_no_memory(-1) < 0
            assert st in (0, kvq.KVQ_ERR_CAPACITY)
            if st:
                assert pages(x.h) == was
                assert _steps(x)[i]() == 0
            assert x.decode() == 0
            if not reached or st or x.plan().any():
                np.testing.assert_array_equal(x.plan(), plan)
            lib.kvq_destroy_cache(x.h)
            if not reached:
                break
        else:
            raise AssertionError("more than 200 allocations")
    d = kvq.kvq_cache_desc(fmt=kvq.KVQ_FMT_AFFINE, key_bits=4, value_bits=4, group_size=32, batch=B, kv_heads=2,
                           q_heads=8, head_dim=64, max_tokens=4096, dtype=kvq.KVQ_BF16,
                           layout=kvq.KVQ_LAYOUT_PAGED, num_pages=60)
    for k in range(50):
        h = ctypes.c_void_p()
        lib.fake_no_memory(k)
        st = lib.kvq_create_cache(ctypes.byref(d), 1 << 32, lib.kvq_cache_bytes(ctypes.byref(d)), ctypes.byref(h))
        reached = lib.fake_no_memory(-1) < 0
        assert (st == kvq.KVQ_ERR_CAPACITY and not h.value) if reached else st == 0
        if not reached:
            break
    assert 3 <= k < 50


@pytest.mark.parametrize("part", [b"copy", b"seq_counts", b"pack_pertoken", b"seq_advance"])
@pytest.mark.parametrize("after", [0, 1])
def test_a_failed_append_gives_its_pages_back(lib, part, after):
    """Pages whose entries may not have reached the table are no sequence's; the next append takes
    them anew and sends their entries."""
    from paper_2609_04263_gb300 import kvq
    x = Host(lib)
    assert x.append([300, 0, 10, 0, 0]) == 0

    def pages():
        return (lib.kvq_free_pages(x.h), [lib.kvq_seq_pages(x.h, b, None, 0) for b in range(B)],
                [lib.kvq_seq_tokens(x.h, b) for b in range(B)])
    was = pages()
    lib.fake_fail(part, after)
    st = x.append([300, 600, 0, 1, 0])
    lib.fake_fail(b"", -1)
    if st == 0:                               # (the kernel is launched once)
        assert after == 1 and part != b"copy"
    else:
        assert st == kvq.KVQ_ERR_CUDA and pages() == was
        assert x.append([300, 600, 0, 1, 0]) == 0
    assert pages() == (60 - 8, [3, 3, 1, 1, 0], [600, 600, 10, 1, 0])
    lib.kvq_destroy_cache(x.h)
