"""KIVI windows whose slots lie more than 2^31 bytes and elements from their start: forks of them, and
decode attention over them."""
import gc

import pytest
import torch

from paper_2609_04263_gb300 import kvq
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture(autouse=True)
def _no_graph_left():
    """Graphs that caught exceptions' frames still hold are freed here: freed in the middle of another
    capture, they would end that one."""
    gc.collect()


def test_a_window_of_more_than_2_to_the_24_tokens():
    from paper_2609_04263_gb300 import api
    D, R, T = 128, 16_800_000, 16_800_010     # (2^31 elements: slot 16,777,216)
    c = api.Cache(api.make_desc(kvq.KVQ_FMT_KIVI, 2, 2, 32, 2, 1, 4, D, T + 100, torch.bfloat16, residual_tokens=R,
                                layout=kvq.KVQ_LAYOUT_PAGED, num_pages=2 * (T // 256 + 2)))
    step = 1 << 21
    z = torch.zeros(2, 1, step, D, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, T - 30, step):
        c.append_ragged(z, z, [min(step, T - 30 - lo), 0])
    # the last 30 tokens: one key a head that outweighs all others by e^40 against 1.7e7, its own value
    q = torch.randn(2, 4, 1, D, device="cuda").bfloat16()
    k, v = torch.zeros(2, 1, 30, D, device="cuda"), torch.randn(2, 1, 30, D, device="cuda")
    for h, t in enumerate((3, 11, 12, 29)):
        qh = q[0, h, 0].float()
        k[0, 0, t] = qh / qh.norm() ** 2 * 40 * D ** 0.5
    q[1] = q[0]
    k, v = k.bfloat16(), v.bfloat16()
    c.append_ragged(k, v, [30, 0])
    c.fork([0], [1])
    planes = c.planes()
    for name, x in (("k_full", k), ("v_full", v)):
        p = planes[name]
        for b in (0, 1):
            assert torch.equal(p[b, 0, T - 30:T], x[0, 0]), (name, b)
    assert torch.equal(planes["k_full"][0, 0, :T], planes["k_full"][1, 0, :T])
    out = c.attend_decode_shared(q).float()
    for b in (0, 1):
        for h, t in enumerate((3, 11, 12, 29)):
            # (keys of other heads' tokens score at most a few; weights below e^-20 of 1.7e7 tokens)
            assert (out[b, h, 0] - v[0, 0, t].float()).abs().max() < 2e-2
