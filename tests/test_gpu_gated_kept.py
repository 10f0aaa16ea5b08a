"""bf16 gated layers: what is kept for the backward pass, 12 significant bits of each factor, and what becomes of it.  Units: f = 2^-24,
k = 2^-12 (half a step of 12 bits).  z, the activation and its slope are off as in test_gpu_gated.py."""
import pytest

from test_gpu_gated import F, _act, _check, _inputs, _run

pytestmark = pytest.mark.gpu
KEPT = 2.0 ** -12


def _bias_gradient(x, dy, w, b, act):
    """Its value and bound in fp64: no rounding but that of the kept factors, of the fp32 products with dy, and of their sum."""
    import torch
    d = w.shape[1]
    x, dy, w, b = x.double().view(-1, d), dy.double().view(-1, w.shape[0] // 2), w.double(), b.double()
    rows = x.shape[0]
    z = x @ w.t() + b
    ez = (d + 2) * F * (x.abs() @ w.abs().t() + b.abs())
    gate, up, eg, eu = z[:, 0::2], z[:, 1::2], ez[:, 0::2], ez[:, 1::2]
    a, slope = _act(gate, act)
    evaluated = 16 * F * (1 + gate.abs())
    ea, es = 1.13 * eg + evaluated, 0.8 * eg + evaluated
    c = up * slope
    ec = up.abs() * es + (slope.abs() + es) * eu + 2 * F * c.abs()
    both = lambda p, q: torch.stack([p, q], 2).view(rows, -1)
    dz = both(dy * c, dy * a)
    edz = both(dy.abs() * ec, dy.abs() * ea) * (1 + KEPT) + (KEPT + F) * dz.abs()
    return dz.sum(0), edz.sum(0) + (rows + 8) * F * dz.abs().sum(0)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,d,f", [(1, 64, 48), (1, 33, 21), (1, 512, 1408), (2, 40, 130), (3, 96, 250), (40, 64, 64), (300, 72, 100)])
def test_bias_gradients_are_sums_of_unrounded_products(rows, d, f, act):
    x, dy, w, b = _inputs(1, rows, d, f, "bf16")
    _check(_run(x, dy, w, b, act, "bf16", rows), {"db": _bias_gradient(x, dy, w, b, act)}, act)
