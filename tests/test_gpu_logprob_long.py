"""Rows longer than a workgroup holds (65527 classes in bf16, 65531 in fp32), most of whose classes are unlikely ones: each adds less to the
sum of exponentials than a step of what the first ones make.

Bounds, f = 2^-24: the maximum is 0, so the likely classes' exponentials are 1 exactly; the others', all alike, are off by (25 + 2) f of
themselves and make up less than 2^-6 of the sum: f at most.  Sums: eight values at a time, then up to 2^18 classes in 256 threads, then 64 lanes and
four waves: 8 + 16 roundings.  Together s = 26 f with the logarithm's; log probabilities s + f |l| (stored)."""
import pytest

from test_gpu_logprob import F, U, _row_parts, _stage

pytestmark = pytest.mark.gpu
SUM = 26 * F


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [65536, 131072, 200003, 262144])
@pytest.mark.parametrize("likely", [1, 256, 700])
def test_many_unlikely_classes(classes, likely, dtype):
    import torch
    rows = 6
    st = _stage(dtype, rows, 1, classes)
    z = torch.full((rows, classes), -17.25, dtype=st.tdtype, device="cuda")   # e^-17.25 is 0.54 of 2^-24
    z[:, :likely] = 0
    ids = torch.tensor([0, classes - 1, -1, likely, 0, classes // 2], dtype=torch.int32, device="cuda")
    soft, logp, one, _, _ = _row_parts(z, ids)
    bound = SUM + F * logp.abs() + 30 * F * (logp < -10)      # the class's own exponent
    got = st.logprobs(z, ids).double()
    print("log probabilities", ((got - logp).abs() / bound).max().item())
    assert bool(((got - logp).abs() <= bound).all()), (got, logp)
    # ratios of one: the slope of a row is -advantage / rows
    adv = torch.tensor([1.0, 1.0, 1.0, 1.0, -1.0, 1.0], device="cuda")
    loss, grad, stored = st.loss_policy(0, z, ids, logp.float(), adv)
    assert torch.equal(stored.double(), got)
    slope = torch.where(ids >= 0, -adv.double() / rows, 0.0)[:, None]
    want = slope * (one - soft)
    # the slope: a ratio is off by what l is, and by f |l| of the stored old one
    allowed = slope.abs() * (one + soft) * (bound + F * logp.abs() + SUM + 8 * F)[:, None] + 30 * F * slope.abs() * soft + U[dtype] * want.abs() + 2.0 ** -126
    over = ((grad.double().view(want.shape) - want).abs() / allowed).max().item()
    print("gradient", over)
    assert over <= 1.0
    pair_ref = torch.zeros(rows, device="cuda")
    assert torch.equal(st.loss_preference(0, z, ids, pair_ref)[2].double(), got)
    st.close()
