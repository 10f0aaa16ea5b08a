"""Rotary positions of short tokens, many of them to a workgroup, and of heads whose parts are units of 8 bytes; bounds as in test_gpu_rotary.py."""
import pytest

from test_gpu_rotary import _compare, _inputs, _spec, _stage

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,spec", [
    (60, _spec(301, heads=1, kv=1, head=16, rotated=8, layout="pairs")), (60, _spec(3001, heads=2, kv=2, head=16, rotated=8)),
    (7, _spec(2999, heads=1, kv=1, head=4, rotated=4, layout="pairs", first=77)), (5, _spec(5000, heads=1, kv=1, head=8, rotated=8)),
    (3, _spec(4001, heads=3, kv=1, head=12, rotated=8)), (2, _spec(2051, heads=4, kv=2, head=80, rotated=40)),
    (1, _spec(1024, heads=2, kv=1, head=20, rotated=16)), (9, _spec(700, heads=2, kv=1, head=36, rotated=28, layout="pairs", factor=2.0, original=128, low=1.0, high=4.0)),
    (1, _spec(2000, heads=1, kv=1, head=256, rotated=256)), (2, _spec(1100, heads=1, kv=1, head=6, rotated=4)), (1, _spec(1500, heads=5, kv=5, head=4, rotated=2, layout="pairs"))],
    ids=lambda s: str(s) if isinstance(s, int) else "-".join(str(v) for v in list(s.__dict__.values())[:-2]))
def test_against_fp64(seqs, spec, dtype):
    import torch
    x, dy = _inputs(spec, seqs, dtype)
    for shift in (0, 4, 2):                                # values by which tensors are off a 16-byte address: whole units, 8-byte ones, neither
        at = lambda t: torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")[shift: shift + t.numel()].view(t.shape).copy_(t)
        st = _stage([spec], dtype, seqs)
        y, dx = at(torch.zeros_like(x)), at(torch.zeros_like(x))
        st.forward(0, 0, at(x), y)
        st.backward(0, at(dy), dx)
        _compare(spec, x, y, False, dtype, shift)
        _compare(spec, dy, dx, True, dtype, shift)
        st.close()
