"""As many sequences as a cache holds, and more of them than a launch's list: forks, copies, roll-backs
and compaction against a model of the page lists and the source's rows, attention against
the calls by sequence."""
import numpy as np
import pytest
import torch

from paper_2609_04263_gb300 import kvq
from tests.gpu_common import require_gpu
from tests.test_gpu_ragged import _seq_rows

pytestmark = pytest.mark.gpu
B, H, HQ, D = 512, 1, 2, 64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _cache(fmt, layout=kvq.KVQ_LAYOUT_PAGED, pages=3000):
    from paper_2609_04263_gb300 import api
    return api.Cache(api.make_desc(fmt, 2, 2, 32, B, H, HQ, D, 1300, torch.bfloat16,
                                   residual_tokens=40 if fmt == kvq.KVQ_FMT_KIVI else 0, layout=layout,
                                   num_pages=pages if layout == kvq.KVQ_LAYOUT_PAGED else 0))


def _rows(c, b):
    T = c.seq_tokens(b)
    coded = max(T - 40, 0) // 32 * 32 if c.desc.fmt == kvq.KVQ_FMT_KIVI else T
    out = {}
    for name in c.planes():
        if name.startswith("_") or name == "workspace":
            continue
        r = _seq_rows(c, name, b, T)
        if name.endswith("_full"):
            out[name] = r[:, :, [t % 72 for t in range(coded, T)]]
        else:
            per = 32 if c.desc.fmt == kvq.KVQ_FMT_KIVI and name in ("k_scale", "k_zero") else 1
            out[name] = r[:, :, :coded // per]
    return {n: r.contiguous().view(torch.uint8) for n, r in out.items()}


def _same_rows(c, b, other, a):
    x, y = _rows(c, b), _rows(other, a)
    for name in x:
        assert torch.equal(x[name], y[name]), (name, b)


def _same_attention(c, n):
    """Both calls lie within 2e-2 of the definition; the two prefills, whose roundings are the same
    (bf16 of the result, fp16 of P and V), each within 0.0024 of its norm."""
    g = torch.Generator(device="cuda").manual_seed(5)
    L = max(n)
    q = torch.randn(B, HQ, L, D, device="cuda", generator=g).bfloat16()
    one = q[:, :, :1].contiguous()
    assert (c.attend_decode_shared(one).float() - c.attend_decode(one).float()).abs().max() < 4e-2
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    c.attend_prefill_shared(q, out=a)
    c.attend_prefill(q, out=b)
    a, b = a.float(), b.float()
    assert (a - b).abs().max() < 4e-2
    for i in range(B):
        x, y = a[i, :, :n[i]], b[i, :, :n[i]]
        assert (x - y).norm() <= 0.0048 * y.norm(), i


@pytest.mark.parametrize("fmt", [kvq.KVQ_FMT_AFFINE, kvq.KVQ_FMT_KIVI, kvq.KVQ_FMT_SYMMETRIC])
def test_all_sequences_of_a_cache(fmt):
    c = _cache(fmt)
    g = torch.Generator(device="cuda").manual_seed(1)

    def append(n):
        k, v = torch.randn(2, B, H, max(n), D, device="cuda", generator=g).bfloat16()
        c.append_ragged(k.contiguous(), v.contiguous(), n)

    append([900] + [0] * (B - 1))
    c.fork([0] * (B - 1), list(range(1, B)))
    for b in (1, 255, 256, 257, 511):
        _same_rows(c, b, c, 0)
    n = [1 + b % 7 for b in range(B)]
    append(n)
    _same_attention(c, n)
    # a second level: eight groups fork their first, each behind tokens of its own
    lead = list(range(0, B, 64))
    append([300 if b in lead else 0 for b in range(B)])
    rest = [b for b in range(B) if b not in lead]
    c.fork([b // 64 * 64 for b in rest], rest)
    for b in (1, 63, 65, 448 + 63):
        _same_rows(c, b, c, b // 64 * 64)
    n = [1 + b % 3 for b in range(B)]
    append(n)
    _same_attention(c, n)
    # into another cache and back over a compacted pool
    other = _cache(fmt, kvq.KVQ_LAYOUT_RAGGED)
    other.copy_from(c, list(range(B)), list(range(B))[::-1])
    for b in (0, 1, 200, 511):
        _same_rows(other, B - 1 - b, c, b)
    c.truncate(list(range(0, B, 2)), [0] * (B // 2))
    c.compact()
    held = {p for b in range(B) for p in c.seq_pages(b)}
    assert held == set(range(len(held))) and c.free_pages() == 3000 - len(held)
    c.copy_from(other, list(range(B - 1, 0, -2)), list(range(0, B, 2)))
    for b in (0, 1, 2, 3, 300, 511):
        _same_rows(c, b, other, B - 1 - b)
    n = [2] * B
    append(n)
    _same_attention(c, n)


def test_each_sequence_cuts_its_copy_of_one_page():
    """512 holders of one page cut inside it: 511 copies, and the last holder keeps it."""
    c = _cache(kvq.KVQ_FMT_AFFINE, pages=1030)
    k = torch.randn(B, H, 512, D, device="cuda").bfloat16()
    c.append_ragged(k, k.flip(2).contiguous(), [512] + [0] * (B - 1))
    ref = _cache(kvq.KVQ_FMT_AFFINE, pages=10)
    ref.append_ragged(k, k.flip(2).contiguous(), [512] + [0] * (B - 1))
    c.fork([0] * (B - 1), list(range(1, B)))
    assert c.free_pages() == 1028
    cut = [257 + b % 200 for b in range(B)]
    c.truncate(list(range(B)), cut)
    assert c.free_pages() == 1030 - 1 - B
    assert len({c.seq_pages(b)[1] for b in range(B)}) == B
    assert len({c.seq_pages(b)[0] for b in range(B)}) == 1
    for b in (0, 1, 2, 100, 510, 511):
        x, y = _rows(c, b), _rows(ref, 0)
        for name in x:
            assert torch.equal(x[name], y[name][:, :, :cut[b]]), (name, b)
    q = torch.randn(B, HQ, 1, D, device="cuda").bfloat16()
    a, b = c.attend_decode_shared(q).float(), c.attend_decode(q).float()
    np.testing.assert_array_less((a - b).abs().max().item(), 4e-2)
