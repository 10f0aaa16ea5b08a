"""Distillation over more rows than one launch has threads for (2^32 of them, 64 or more to a row)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [1])
def test_more_rows_than_a_launch_takes(k):
    """2^26 rows and some, a wave each.  Bounds as in test_gpu_distill.py: probabilities of 16 classes, exponents up to 6, are off by 64 x 2^-24 of
    themselves, the stored gradient by 2^-8, the loss, whose rows are added up in 64 bits, by 64 x 2^-24 (1 + 6)."""
    import torch
    from paper_2509_23241_amd import binding as B
    from paper_2509_23241_amd.runner import GpuStage
    classes, mb, tokens, t = 16, 64, (1 << 20) + 3, 2.0
    rows = mb * tokens
    st = GpuStage([(8, classes, "none", tokens)], [np.zeros((classes, 8), np.float32), np.zeros(classes, np.float32)], dtype="bf16", mb=mb, n=1,
                  stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0, ring_capacity=1, max_in_flight=1)
    st.forward(0, 0, torch.zeros(mb, 8 * tokens, dtype=torch.bfloat16, device="cuda"))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    z = torch.randn(rows, classes, generator=g, device="cuda", dtype=torch.bfloat16)
    teacher = torch.zeros(rows, k, device="cuda")
    ids = torch.zeros(rows, k, dtype=torch.int32, device="cuda")
    out = torch.full_like(z, 7.0)
    loss = torch.empty(1, device="cuda")
    B.stage_loss_distill(st.handle, 0, z.data_ptr(), teacher.data_ptr(), ids.data_ptr(), k, t, 0, 0.0, out.data_ptr(), loss.data_ptr())
    torch.cuda.synchronize()
    total = 0.0
    for a in range(0, rows, 1 << 22):
        b = slice(a, min(a + (1 << 22), rows))
        logq = (z[b].double() / t).log_softmax(1)
        want = logq.exp()
        want[:, 0] -= 1
        size = (logq.exp() + (torch.arange(classes, device="cuda") == 0)) * (t / rows)
        want *= t / rows
        off = (out[b].double() - want).abs()
        assert bool((off <= 64 * 2.0 ** -24 * size + 2.0 ** -8 * (want.abs() + 64 * 2.0 ** -24 * size)).all()), a
        total += float(-t * t * logq[:, 0].sum())
    assert abs(float(loss) - total / rows) <= 64 * 2.0 ** -24 * 7 * t * t
    st.close()
