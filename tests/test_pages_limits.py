"""Sizes that 32 bits cannot count, refused where a paged cache is made, and other
arguments that no kernel could work with (no GPU)."""
import pytest

from tests.test_pages_abi import P, _cache, _refused, kvq, paged  # noqa: F401  (fixtures)


@pytest.mark.parametrize("kw", [dict(num_pages=1 << 23), dict(num_pages=2 ** 31 - 1),
                                dict(batch=512, max_tokens=1 << 30), dict(max_tokens=2 ** 31 - 1),
                                dict(max_tokens=2 ** 31 - 255)])
def test_pools_and_tables_too_large_to_count(kvq, kw):  # noqa: F811
    _refused(kvq, kvq.KVQ_ERR_SHAPE, lambda: _cache(kvq, **kw))


@pytest.mark.parametrize("kw,gib", [(dict(num_pages=(1 << 23) - 1), 2 ** 31 * 2 * (32 + 4 + 4) * 2 / 2 ** 30),
                                    (dict(batch=512, max_tokens=(1 << 30) - 512), 8)])
def test_the_largest_that_can_be_counted(kvq, kw, gib):  # noqa: F811
    """2^31 - 256 rows of 2 heads, 32 + 4 + 4 bytes a row for keys and for values; 2^31 entries of 4 bytes."""
    d = dict(fmt=kvq.KVQ_FMT_AFFINE, key_bits=4, value_bits=4, group_size=32, residual_tokens=0, sink_tokens=0,
             norm_iters=8, batch=4, kv_heads=2, q_heads=8, head_dim=64, max_tokens=1000, dtype=kvq.KVQ_BF16,
             layout=kvq.KVQ_LAYOUT_PAGED, num_pages=9)
    d.update(kw)
    n = kvq.kvq_cache_bytes(kvq.kvq_cache_desc(**d)) / 2 ** 30
    assert gib * 0.999 < n < gib * 1.1


@pytest.mark.parametrize("scale", [2.4e38, 3.0e38, 3.4e38])
def test_scales_that_overflow_in_log2_units(kvq, paged, scale):  # noqa: F811
    n = kvq.kvq_attend_shared_workspace(paged, 1)
    _refused(kvq, kvq.KVQ_ERR_ARG, kvq.kvq_attend_decode_shared, paged, P, 8, scale, P, P, n)
    _refused(kvq, kvq.KVQ_ERR_ARG, kvq.kvq_attend_prefill_shared, paged, P, 1, 8, scale, P, P, n)


def test_lists_that_the_call_would_read_past(kvq, paged):  # noqa: F811
    """The binding gives one count: that of the other lists is checked."""
    for call, args in ((kvq.kvq_seq_fork, ([0], [1, 2])), (kvq.kvq_seq_fork, ([0, 0], [1, 2], [0])),
                       (kvq.kvq_seq_copy, (paged, [0], [1, 2])), (kvq.kvq_seq_copy, (paged, [0, 0], [1, 2], [0])),
                       (kvq.kvq_seq_truncate, ([0, 1], [0])), (kvq.kvq_seq_truncate, ([], [0]))):
        with pytest.raises(ValueError):
            call(paged, *args)


def test_an_append_needs_a_count_a_sequence(kvq):  # noqa: F811
    import types

    from paper_2609_04263_gb300 import api
    cache = types.SimpleNamespace(desc=types.SimpleNamespace(batch=4), handle=None)
    for n in ([], [1], [1] * 5):
        with pytest.raises(ValueError):
            api.Cache.append_ragged(cache, None, None, n)
