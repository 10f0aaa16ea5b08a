"""Windowed attention layers with many heads to a key head are taken whatever their buckets; no GPU needed."""
import pytest

from paper_2509_23241_amd import binding as B


def _query(layer, dtype, **changed):
    given = dict(dtype=dtype, mb=2, n=3, stage_index=1, num_stages=4, ring_capacity=3, max_in_flight=3, policy="convex", needs_dx=True,
                 lam=0.1, lr=0.01, momentum=0.9)
    return B.stage_workspace_query(B.make_desc([layer], **{**given, **changed}))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_heads_and_buckets(dtype):
    for heads, dh, buckets in ((64, 128, 128), (128, 192, 128), (256, 256, 128), (1000, 3, 128), (65535, 1, 2)):
        s = _query(("local", heads * dh, heads, 8, 1, 3, 1, buckets, 900), dtype)
        assert s.param_count >= heads * buckets


def test_more_heads_than_a_grid_has_rows():
    with pytest.raises(B.StageLibError) as e:
        _query(("local", 65536, 65536, 8, 1, 3, 1), "bf16")
    assert e.value.code == B.TP_EINVAL


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_numbers_of_tokens_next_to_the_limits(dtype):
    """2^23 blocks of 16 tokens and no more, up to the largest number a description holds."""
    for tokens, mb in ((1 << 27, 1), (1 << 24, 8), (16, 1 << 23)):
        _query(("local", 4, 4, tokens, 2, 3, 1), dtype, mb=mb, n=1)
    for tokens, mb in (((1 << 27) + 1, 1), ((1 << 24) + 1, 8), (17, 1 << 23), ((1 << 31) - 16, 1), ((1 << 31) - 15, 1), ((1 << 31) - 1, 1),
                       ((1 << 31) - 1, 1 << 24)):
        with pytest.raises(B.StageLibError) as e:
            _query(("local", 4, 4, tokens, 2, 3, 1), dtype, mb=mb, n=1)
        assert e.value.code == B.TP_EINVAL, (tokens, mb)
