"""Gated layers whose fp32 operands are copied into rows of whole 16-byte units (widths that are no multiple of four, 256 rows and more), whose
gradients are summed over ranges of their contraction, and what stands next to them; bounds as in test_gpu_gated.py."""
import numpy as np
import pytest

from test_gpu_gated import _check, _inputs, _reference, _run, _stage

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,tokens,d,f", [(1, 255, 130, 66), (1, 256, 130, 66), (1, 256, 3, 5), (1, 700, 101, 259), (2, 500, 999, 300), (1, 300, 1500, 400),
                                             (1, 321, 64, 1500), (1, 260, 67, 2050), (1, 3000, 33, 31), (5, 200, 258, 129)])
def test_against_fp64(seqs, tokens, d, f, dtype):
    x, dy, w, b = _inputs(seqs, tokens, d, f, dtype)
    for shift in (0, 1):
        _check(_run(x, dy, w, b, "silu", dtype, tokens, shift=shift), _reference(x, dy, w, b, "silu", dtype), shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,f", [(130, 66), (67, 300)])
def test_micro_batches_and_streams_give_the_same_bits(d, f, dtype):
    import torch
    x, dy, w, b = _inputs(6, 100, d, f, dtype)
    whole = _run(x, dy, w, b, "gelu", dtype, 100)
    for other in (_run(x, dy, w, b, "gelu", dtype, 100, n=3), _run(x, dy, w, b, "gelu", dtype, 100, n=3, minibatch=True)):
        for k in whole:
            assert torch.equal(whole[k], other[k]), k
    st = _stage([("gated", d, f, "gelu", 100)], [w.cpu().numpy(), b.cpu().numpy()], dtype, 2, 3, forward_stream=3)
    for _ in range(2):                                     # the second time with what the first has left in the copies
        y, dx = torch.empty_like(dy), torch.empty_like(x)
        for ub in range(3):
            st.forward(_, ub, x[2 * ub: 2 * ub + 2], y[2 * ub: 2 * ub + 2])
        st.backward(_, dy, dx)
        st.blend_update(_)
        assert torch.equal(y.view(-1, f), whole["y"]) and torch.equal(dx.view(-1, d), whole["dx"])
    st.close()


def test_layers_beside_it():
    """Behind a ReLU, whose mask the input gradient passes, directly inside a residual connection, in front of and behind layers of odd widths."""
    from stage_parity import run_stage
    from synth_inputs import workloads as W
    t = 80
    for dtype in ("f32", "bf16"):
        specs = (W.Dense(16, 67, "relu", tokens=t), W.Gated(67, 700, "silu", t), W.Dense(700, 21, "none", tokens=t), W.LayerNorm(21, t), W.Gated(21, 13, "gelu", t))
        print(dtype, run_stage(specs, f"gated_relu_{dtype}", dtype, mb=2, n=2, policy="convex", fixed_masks=True, mean_loss_dy=True))
        specs = (W.Dense(16, 70, "none", tokens=t), W.Residual(70, t, "begin"), W.Gated(70, 70, "silu", t), W.Residual(70, t, "add"), W.LayerNorm(70, t),
                 W.Dense(70, 9, "none", tokens=t))
        print(dtype, run_stage(specs, f"gated_residual_{dtype}", dtype, mb=2, n=2, policy="convex", mean_loss_dy=True))
