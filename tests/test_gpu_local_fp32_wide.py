"""Windowed attention in fp32 with heads above 64, whose launches are cut up for one workgroup on a CU, against fp64 within the bounds of
test_gpu_local_attention.py: sizes that fill the chip, that do not, and that take parts of a walk."""
import pytest

from test_gpu_local_attention import _case, _check, _inputs, _reference, _run

pytestmark = pytest.mark.gpu

CASES = [_case(300, heads=8, kv=8, dh=128, seqs=8), _case(1500, heads=4, kv=1, dh=128, window=400, seqs=1),
         _case(1100, heads=4, kv=1, dh=96, window=300, sinks=5, buckets=20, reach=500, seqs=1), _case(260, heads=8, kv=8, dh=80, window=60, sinks=2, seqs=16),
         _case(700, heads=2, kv=2, dh=128, buckets=16, reach=300, seqs=2), _case(600, heads=16, kv=2, dh=72, window=90, sinks=40, seqs=1)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in list(c.values())[:-1]))
def test_against_fp64(case):
    c = dict(case, dtype="f32")
    x, dy, table = _inputs(c)
    _check(_run(c, x, dy, table), _reference(c, x, dy, table))
