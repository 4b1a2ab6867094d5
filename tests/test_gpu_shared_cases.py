"""The performance cases of shared pages (perf/operators.py): the package's calls and the plain form
on the same inputs.  Copies agree bit for bit; attention lies within 0.0024 of the norm of the
definition in 64 bits on both sides (bf16's rounding of the result, 2^-8 / sqrt(3) = 0.00226 root mean
square, and P and V in fp16, below 0.0005), which it did not where the two sides coded the same
tokens by different quotients."""
import importlib.util
import os
import random

import pytest
import torch

from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture
def cases():
    spec = importlib.util.spec_from_file_location("performance_cases", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _outputs(cases, case, own, seed):
    cases.own = own
    out = cases.run(cases.prepare(case, seed))
    torch.cuda.synchronize()
    return out if isinstance(out, list) else [out]


def _small(case):
    tokens = case.get("root", case.get("tokens")) + case.get("branch", 0)
    return tokens * case.get("batch", case.get("copies", 1)) < 300_000


def _check(cases, case, seed):
    plain, own = (_outputs(cases, case, x, seed) for x in (False, True))
    if case["op"] not in ("decode", "prefill"):
        for x, y in zip(plain, own):
            # (bits: planes hold random fp16 words, NaN among them)
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
        return
    ref = cases.exact(case, seed)
    for x in (plain[0], own[0]):
        assert (x.double() - ref).norm() <= 0.0024 * ref.norm()


@pytest.mark.parametrize("name", ["fork_small", "fork_samples_kivi", "decode_small", "decode_16_kivi",
                                  "decode_tree_sym", "decode_mha_affine", "prefill_verify_affine",
                                  "prefill_questions_affine"])
def test_listed_cases(cases, name):
    _check(cases, next(c for c in cases.listed() if c["name"] == name), 3)


def test_drawn_cases(cases):
    rng = random.Random(21)
    small = [c for c in (cases.draw(rng) for _ in range(60)) if _small(c)][:12]
    assert {c["op"] for c in small} >= {"fork", "decode", "prefill"}
    for i, case in enumerate(small):
        _check(cases, case, i)
