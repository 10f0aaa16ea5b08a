"""Rows without stored entries where the teacher alone counts: padded positions of a batch, whose logits may hold anything."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [5, 20, 700, 1500, 40001, 140000])
def test_rows_without_a_term_have_no_gradient(classes, dtype):
    import torch
    from paper_2509_23241_amd.runner import GpuStage
    rows, k = 9, 3
    st = GpuStage([(8, classes, "none")], [np.zeros((classes, 8), np.float32), np.zeros(classes, np.float32)], dtype=dtype, mb=rows, n=1,
                  stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0, ring_capacity=1, max_in_flight=1)
    st.forward(0, 0, torch.zeros(rows, 8, dtype=st.tdtype, device="cuda"))
    g = torch.Generator(device="cuda")
    g.manual_seed(classes)
    z = torch.randn(rows, classes, generator=g, device="cuda").to(st.tdtype)
    ids = torch.rand(rows, classes, generator=g, device="cuda").topk(k, 1).indices.to(torch.int32)
    teacher = torch.randn(rows, k, generator=g, device="cuda")
    empty = [1, 2, 4, 6, 8]
    ids[[1, 2, 4]] = -1
    teacher[[6, 8]] = -np.inf
    clean = [t.clone() for t in st.loss_distill(0, z, teacher, ids, temperature=2.0)]
    for value in (np.nan, np.inf, -np.inf):
        for whole in (True, False):
            bad = z.clone()
            bad[empty] = value if whole else bad[empty]
            bad[empty, 1] = value
            for t in (1.0, 2.0):
                loss, grad = st.loss_distill(0, bad, teacher, ids, temperature=t)
                assert bool((grad[empty] == 0).all()) and np.isfinite(float(loss)), (value, whole, t)
            assert torch.equal(loss, clean[0]) and torch.equal(grad, clean[1])
    # a label is a term: what its row holds arrives
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    bad = z.clone()
    bad[1, 1] = np.nan
    loss, grad = st.loss_distill(0, bad, teacher, ids, temperature=2.0, labels=labels, label_weight=0.5)
    assert np.isnan(float(loss)) and bool(torch.isnan(grad[1]).any()) and bool(torch.isfinite(grad[[0, 2, 3]]).all())
    st.close()
