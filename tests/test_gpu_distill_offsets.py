"""Distillation from stored logits where a row's logits lie far from zero: a softmax does not depend on what all of them have in common, and
neither may its error.

Bounds, unit f = 2^-24.  An exponent x / a (a: the temperature, or 1 for the labels' softmax), x the distance from the row's maximum, is off by at
most 4 f of itself: the scale, the temperature, the difference and a product.  An exponential: that and 2 f; a sum of n of them: `chain` =
min(n, 64) + 22 + n / 256 roundings of a thread, its wave and its workgroup; a logarithm 2 f (1 + log2 n).  None of it knows the offset."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
F = 2.0 ** -24


def _stage(dtype, rows, classes):
    import torch
    from paper_2509_23241_amd.runner import GpuStage
    st = GpuStage([(8, classes, "none")], [np.zeros((classes, 8), np.float32), np.zeros(classes, np.float32)], dtype=dtype, mb=rows, n=1,
                  stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0, ring_capacity=1, max_in_flight=1)
    st.forward(0, 0, torch.zeros(rows, 8, dtype=st.tdtype, device="cuda"))
    return st


def _want(z, teacher, ids, t, labels, w):
    """Loss and gradient in fp64 and what they may be off by."""
    import torch
    rows, n = z.shape
    k = ids.shape[1]
    z = z.double() - z.double().amax(1, keepdim=True)
    x = teacher.double() / t
    logp = x - x.logsumexp(1, keepdim=True)
    p, at, label = logp.exp(), ids.long(), labels.long()[:, None]
    logq, logs = (z / t).log_softmax(1), z.log_softmax(1)
    ratio = logp - logq.gather(1, at)
    c = (1 - w) * t
    loss = w * -logs.gather(1, label)[:, 0] + c * t * (p * ratio).sum(1)
    scatter = torch.zeros_like(z).scatter_add_(1, at, p)
    one = torch.zeros_like(z).scatter_(1, label, 1.0)
    q, s = logq.exp(), logs.exp()
    grad = (c * (q - scatter) + w * (s - one)) / rows
    spread, tspread, log = float(-z.min()), float(teacher.max() - teacher.min()), 2 * (1 + math.log2(n))
    chain = min(n, 64) + 22 + n / 256
    off_s, off_q, off_p = chain + 2 + 4 * spread, chain + 2 + 4 * spread / t, k + 10 + 8 * tspread / t
    eloss = (w * (off_s + log + 4 * float((-logs).gather(1, label).max())) +
             c * t * (off_q + log + off_p * (1 + float(ratio.abs().max())))) * F
    egrad = (c * (q * (off_q + 4 * spread / t + 8) + scatter * (off_p + 8)) + w * (s * (off_s + 4 * spread + 8) + one * 8)) * F / rows
    return float(loss.mean()), grad, eloss, egrad


@pytest.mark.parametrize("dtype,offset,step", [("f32", 0, 0.25), ("f32", 100, 0.25), ("f32", 1003, 0.25), ("f32", 10007, 0.25), ("f32", -10007, 0.25),
                                               ("bf16", 100, 0.5), ("bf16", 1004, 4.0), ("bf16", -1004, 4.0), ("bf16", 10048, 64.0)])
@pytest.mark.parametrize("classes", [20, 1500, 40001, 140000])
def test_the_error_does_not_grow_with_what_all_logits_have_in_common(classes, dtype, offset, step):
    import torch
    rows, k = 6, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(classes)
    z = offset + step * torch.randint(-3, 1, (rows, classes), generator=g, device="cuda").double()
    ids = torch.rand(rows, classes, generator=g, device="cuda").topk(k, 1).indices.to(torch.int32)
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    rowsat = torch.arange(0, rows, 2, device="cuda")
    z[rowsat, labels[::2].long()] = offset + max(16.0, step)        # the label has nearly all the probability
    stored = z.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    assert bool((stored.double() == z).all())
    teacher = torch.randn(rows, k, generator=g, device="cuda")
    st = _stage(dtype, rows, classes)
    for t, w in ((1.5, 0.9375), (3.0, 0.9375), (0.7, 0.5), (3.0, 0.0), (1.0, 0.5), (3.0, 1.0)):
        loss, grad = st.loss_distill(0, stored, teacher, ids, temperature=t, labels=labels, label_weight=w)
        want, dwant, eloss, egrad = _want(z, teacher, ids, t, labels, w)
        off = abs(float(loss) - want)
        bound = egrad + (2.0 ** -8 if dtype == "bf16" else F) * (dwant.abs() + egrad) + 2.0 ** -126
        share = float(((grad.double() - dwant).abs() / bound).max())
        print("T", t, "w", w, "loss off %.1e of %.1e" % (off, eloss + F * abs(want)), "gradient %.2f of its bound" % share)
        assert off <= eloss + F * abs(want), (t, w)
        assert share <= 1.0, (t, w)
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 40001, 140000])
@pytest.mark.parametrize("t,offset", [(1e-6, 2000.0), (1e-6, 30000.0), (1e-5, 1e6), (1e-6, -30000.0), (1e-6, 1e12)])
def test_logits_far_beyond_the_temperature(t, offset, classes, dtype):
    """All probability on the largest logit, whatever max / T is rounded by.  The loss of an entry that lies `gap` below is T gap, the gradient
    T on the one class and -T on the other; each is a product of five rounded factors at most."""
    import torch
    rows = 5
    tt = torch.float32 if dtype == "f32" else torch.bfloat16
    base = torch.tensor(offset).to(tt).double()
    step = 2.0 ** (math.floor(math.log2(abs(offset))) - (6 if dtype == "bf16" else 20))
    z = (base - step * (2 + torch.arange(classes).double() % 3)).repeat(rows, 1)
    best, entry = torch.arange(rows) + 3, torch.arange(rows) + 11
    z[torch.arange(rows), best] = base
    z[torch.arange(rows), entry] = base - 3 * step
    stored = z.to(tt)
    assert bool((stored.double() == z).all())
    st = _stage(dtype, rows, classes)
    teacher = torch.zeros(rows, 2, device="cuda")
    ids = torch.stack([entry, torch.full((rows,), -1)], 1).to(torch.int32).contiguous().cuda()
    for w in (0.0, 0.5):
        labels = entry.to(torch.int32).cuda()
        loss, grad = st.loss_distill(0, stored.cuda(), teacher, ids, temperature=t, labels=labels, label_weight=w)
        hard = torch.exp(z - base).sum(1).log() + 3 * step       # of the labels' softmax: the classes within some 100 of the maximum
        want = (1 - w) * t * 3 * step + w * float(hard.mean())
        # chain of its sum and one logarithm, as above, and the exponents of classes that count (within 18 of the maximum)
        eloss = 16 * F * want + w * F * (min(classes, 64) + 24 + classes / 256 + 4 * 18 + 2 * (1 + math.log2(classes)))
        assert abs(float(loss) - want) <= eloss, (w, float(loss), want, eloss)
        if w == 0.0:
            dwant = torch.zeros(rows, classes, dtype=torch.float64)
            dwant[torch.arange(rows), best] = t / rows
            dwant[torch.arange(rows), entry] = -t / rows
            off = (grad.double().cpu() - dwant).abs()
            assert bool((off <= dwant.abs() * (16 * F + (2.0 ** -8 if dtype == "bf16" else 0))).all())
        else:
            assert bool(torch.isfinite(grad).all())
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 40001, 140000])
def test_labels_that_have_nearly_all_the_weight(classes, dtype):
    """What is left for the teacher, 1 - label_weight, is right to a rounding of its own; the label's own term is next to nothing here."""
    import torch
    rows, k = 6, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(classes)
    z = 0.25 * torch.randint(-3, 1, (rows, classes), generator=g, device="cuda").double()
    ids = torch.rand(rows, classes, generator=g, device="cuda").topk(k, 1).indices.to(torch.int32)
    labels = (ids[:, 0] + 1) % classes
    z[torch.arange(rows, device="cuda"), labels.long()] = 64.0
    stored = z.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    teacher = torch.randn(rows, k, generator=g, device="cuda")
    st = _stage(dtype, rows, classes)
    for t, w in ((1.5, 0.999), (3.0, 0.9999), (1.0, 0.9999), (2.0, 1 - 2.0 ** -30)):
        loss, grad = st.loss_distill(0, stored, teacher, ids, temperature=t, labels=labels, label_weight=w)
        want, dwant, eloss, egrad = _want(z, teacher, ids, t, labels, w)
        bound = egrad + (2.0 ** -8 if dtype == "bf16" else F) * (dwant.abs() + egrad) + 2.0 ** -126
        share = float(((grad.double() - dwant).abs() / bound).max())
        print("T", t, "w", w, "loss off %.1e of %.1e" % (abs(float(loss) - want), eloss + F * abs(want)), "gradient %.2f of its bound" % share)
        assert abs(float(loss) - want) <= eloss + F * abs(want), (t, w)
        assert share <= 1.0, (t, w)
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 40001, 140000])
@pytest.mark.parametrize("t,offset", [(1e6, 1e12), (1e6, -1e12), (50.0, 1e10), (1e3, 3e8)])
def test_large_logits_at_high_temperatures(t, offset, classes, dtype):
    """What max / T is rounded by counts T times in the labels' softmax, which has all its probability on the largest logit here: its terms are off by
    8 roundings.  The teacher's are bounded as above."""
    import torch
    rows, k = 5, 4
    tt = torch.float32 if dtype == "f32" else torch.bfloat16
    base = torch.tensor(offset).to(tt).double()
    step = 2.0 ** (math.floor(math.log2(abs(offset))) - (6 if dtype == "bf16" else 20))
    assert step >= 128
    at = torch.arange(rows)
    z = (base - step * (1 + torch.arange(classes).double() % 3)).repeat(rows, 1)
    z[at, at + 3] = base
    stored = z.to(tt)
    assert bool((stored.double() == z).all())
    g = torch.Generator().manual_seed(classes)
    ids = torch.rand(rows, classes, generator=g).topk(k, 1).indices.to(torch.int32).cuda()
    teacher, labels = torch.randn(rows, k, generator=g).cuda(), (at + 5).to(torch.int32).cuda()
    z = z.cuda()
    st = _stage(dtype, rows, classes)
    for w in (0.0, 0.5, 1.0):
        loss, grad = st.loss_distill(0, stored.cuda(), teacher, ids, temperature=t, labels=labels, label_weight=w)
        want, dwant, eloss, egrad = _want(z, teacher, ids, t, labels, w)
        assert abs(float(loss) - want) <= eloss + F * abs(want), w
        if w > 0:   # without the labels' exponents in the bound: their probabilities are 0 and 1
            _, _, _, teachers = _want(z, teacher, ids, t, labels, 0.0)
            egrad = (1 - w) * teachers + w * (dwant != 0) * 8 * F / rows
        bound = egrad + (2.0 ** -8 if dtype == "bf16" else F) * (dwant.abs() + egrad) + 2.0 ** -126
        assert bool(((grad.double() - dwant).abs() <= bound).all()), w
    st.close()
