"""bf16 gated layers: what is kept for the backward pass, 12 significant bits of each factor, and what becomes of it.  Units: f = 2^-24,
k = 2^-12 (half a step of 12 bits).  z, the activation and its slope are off as in test_gpu_gated.py."""
import numpy as np
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


@pytest.mark.parametrize("bits", [0x7fffffff, 0xffffffff, 0x7fc00000, 0xffc00000])
@pytest.mark.parametrize("rows,d,f", [(3, 16, 12), (40, 33, 21), (300, 64, 130)])
def test_a_bias_that_is_no_number_reaches_its_gradients(rows, d, f, bits):
    """NaN of any payload, one with all bits set among them: outputs, gradients and input gradients that hang on it are NaN."""
    import torch
    x, dy, w, b = _inputs(1, rows, d, f, "bf16")
    for column in (4, 7):                                  # a gate; the other factor of another output
        bad = b.clone()
        bad.view(torch.int32)[column] = np.array([bits], np.uint32).view(np.int32).item()
        clean, got = _run(x, dy, w, b, "silu", "bf16", rows), _run(x, dy, w, bad, "silu", "bf16", rows)
        unit = column // 2
        others = torch.arange(f, device="cuda") != unit
        assert bool(torch.isnan(got["y"][:, unit]).all()) and torch.equal(got["y"][:, others], clean["y"][:, others])
        hit = torch.zeros(2 * f, dtype=torch.bool, device="cuda")
        hit[2 * unit] = True                               # dy z_2f+1 act'(z_2f)
        hit[2 * unit + 1] = column == 2 * unit             # dy act(z_2f)
        for k in ("db", "dw"):
            assert bool(torch.isnan(got[k][hit]).all()), (column, k)
            assert torch.equal(got[k][~hit], clean[k][~hit]), (column, k)
        assert bool(torch.isnan(got["dx"]).all())
