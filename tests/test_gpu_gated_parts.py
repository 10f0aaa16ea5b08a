"""fp32 gated layers whose contraction is summed in parts, the last of them short: a product of few tiles, of many, and of an input at an odd
address are formed by three kernels, and leave the same bits."""
import pytest

from test_gpu_gated import _check, _inputs, _reference, _run

pytestmark = pytest.mark.gpu


# rows of a micro-batch: at most 1024 tiles of 16 x 16 outputs, where the whole mini-batch has more
@pytest.mark.parametrize("d,f,rows,n", [(288, 512, 256, 4), (384, 512, 256, 4), (320, 1024, 128, 4), (544, 333, 384, 2), (800, 256, 512, 2),
                                        (383, 512, 256, 2), (992, 128, 1024, 2), (256, 512, 256, 2), (512, 512, 256, 2), (224, 512, 256, 2)])
def test_micro_batches_give_the_same_bits(d, f, rows, n):
    import torch
    x, dy, w, b = _inputs(n, rows, d, f, "f32")
    whole = _run(x, dy, w, b, "silu", "f32", rows)
    _check(whole, _reference(x, dy, w, b, "silu", "f32"))
    for ways in (dict(n=n), dict(n=n, minibatch=True), dict(n=n, shift=1), dict(shift=1)):
        other = _run(x, dy, w, b, "silu", "f32", rows, **ways)
        for k in whole:
            assert torch.equal(whole[k], other[k]), (ways, k, float((whole[k] - other[k]).abs().max()))
