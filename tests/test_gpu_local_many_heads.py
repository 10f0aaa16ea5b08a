"""Windowed attention with many query heads on one key head and many buckets, on the matrix cores and at odd addresses, against fp64 within the
bounds of test_gpu_local_attention.py."""
import numpy as np
import pytest

from test_gpu_local_attention import _case, _check, _inputs, _params, _reference, _run, _split, _stage

pytestmark = pytest.mark.gpu

CASES = [_case(50, heads=64, kv=1, dh=128, window=20, sinks=2, buckets=128, reach=300, seqs=1),
         _case(40, heads=80, kv=1, dh=200, buckets=128, reach=90, seqs=1), _case(35, heads=300, kv=2, dh=12, window=9, buckets=100, reach=70, seqs=1),
         _case(70, heads=96, kv=1, dh=64, window=30, sinks=1, buckets=128, reach=200, seqs=2)]
ids = lambda c: "-".join(str(v) for v in list(c.values())[:-1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_many_heads_of_a_key_head(case, dtype):
    c = dict(case, dtype=dtype)
    x, dy, table = _inputs(c)
    _check(_run(c, x, dy, table), _reference(c, x, dy, table))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_at_any_address(case, dtype):
    import torch
    c = dict(case, dtype=dtype)
    x, dy, table = _inputs(c)
    st = _stage(c, _params(table))
    put = lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(c["seqs"], -1)
    y, dx = put(torch.zeros_like(dy)), put(torch.zeros_like(x))
    st.forward(0, 0, put(x), y)
    st.backward(0, put(dy), dx)
    _check(_split(c, y, dx, st.grad), _reference(c, x, dy, table))
    st.close()


def test_a_workgroup_with_several_blocks_of_rows_adds_them_up():
    """More row blocks than there are rows of partial sums (512): odd widths, so that the kernels for any width take them."""
    for dtype in ("f32", "bf16"):
        c = _case(50, heads=4, kv=2, dh=5, window=20, sinks=1, buckets=16, reach=40, seqs=150, dtype=dtype)
        x, dy, table = _inputs(c)
        _check(_run(c, x, dy, table), _reference(c, x, dy, table))
