"""Distillation from stored top logits (kernels_distill.hip) against fp64: sizes around what a workgroup holds, entries that are
absent, repeated, infinite, or no class, labels, alignment.

Bounds, unit f = 2^-24: an exponent x / T has an error of 4 f (|x / T| + 1) (the difference, the scale, the product), an exponential the
same plus 2 f relative, a sum of n terms over lanes (classes / 256 + 16) f.  So probabilities are off by
(4 (range / T + 1) + classes / 64 + 32) f of themselves, logarithms of them by as much; gradients add one rounding of each term, bf16
ones 2^-8 of the result."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _stage(dtype, rows, classes, tokens=1):
    import torch
    from paper_2509_23241_amd.runner import GpuStage
    st = GpuStage([(8, classes, "none", tokens)], [np.zeros((classes, 8), np.float32), np.zeros(classes, np.float32)], dtype=dtype, mb=rows,
                  n=1, stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0, ring_capacity=1, max_in_flight=1)
    st.forward(0, 0, torch.zeros(rows, 8 * tokens, dtype=st.tdtype, device="cuda"))
    return st


def _reference(z, teacher, ids, t, labels, w):
    """Row losses and the gradient of their mean, and the bounds of both, in fp64 (a class that does not exist: its term left out)."""
    import torch
    z, teacher = z.double(), teacher.double()
    rows, classes = z.shape
    f = 2.0 ** -24
    kept = (ids >= 0) & (teacher > -np.inf)
    there = kept & (ids < classes)
    x = teacher.masked_fill(~kept, -np.inf) / t
    has = kept.any(1, keepdim=True) & (w < 1)
    logp = torch.where(has, x - x.logsumexp(1, keepdim=True), -np.inf)
    p = logp.exp()
    at = ids.long().clamp(0, classes - 1)
    logq = (z / t).log_softmax(1)
    logs = z.log_softmax(1)
    known = (labels >= 0) & (labels < classes)
    label = labels.long().clamp(0, classes - 1)[:, None]
    kl = torch.where((p > 0) & there, p * (logp - logq.gather(1, at)), 0).sum(1)
    loss = (w * -logs.gather(1, label)[:, 0] if w > 0 else 0) + (1 - w) * t * t * kl
    scatter = torch.zeros_like(z).scatter_add_(1, at, p * there)
    one = torch.zeros_like(z).scatter_(1, label, known.double()[:, None])
    c = (1 - w) * t
    q, s = logq.exp() * has, logs.exp()
    grad = (c * (q - scatter) + w * (s - one)) / rows
    finite = z.masked_fill(~torch.isfinite(z), 0)
    spread = float((finite.max() - finite.min()).abs()) + float(teacher.masked_fill(~kept, 0).nan_to_num(0, 0, 0).abs().max())
    off_q, off_s = ((4 * (spread / a + 1) + classes / 64 + 32) * f for a in (t, 1.0))
    egrad = (c * (q + scatter) * (off_q + 8 * f) + w * (s + one) * (off_s + 8 * f)) / rows
    eloss = w * (off_s + 8 * f) * (1 + loss.abs().max()) + (1 - w) * t * t * (off_q + 8 * f) * (2 + spread / t)
    return loss, grad, float(eloss), egrad


def _inputs(dtype, rows, classes, k, seed=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + rows + classes + k)
    tt = torch.float32 if dtype == "f32" else torch.bfloat16
    z = (3 * torch.randn(rows, classes, generator=g, device="cuda")).to(tt)
    ids = torch.rand(rows, classes, generator=g, device="cuda").topk(k, 1).indices.to(torch.int32)
    teacher = 3 * torch.randn(rows, k, generator=g, device="cuda")
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    return z, teacher, ids, labels


def _compare(dtype, z, teacher, ids, labels, t, w, got=None, st=None):
    import torch
    loss, grad, eloss, egrad = _reference(z, teacher, ids, t, labels, w)
    if got is None:
        own = st is None
        st = st or _stage(dtype, *z.shape)
        got = st.loss_distill(0, z, teacher, ids, temperature=t, labels=labels if w > 0 else None, label_weight=w)
        got = got[0].clone(), got[1].clone()
        if own:
            st.close()
    assert abs(float(got[0]) - float(loss.mean())) <= eloss + 2.0 ** -24 * abs(float(loss.mean())), (float(got[0]), float(loss.mean()))
    off = (got[1].double() - grad).abs()
    # a result that is smaller than the smallest normal bf16 or fp32 value has no relative rounding
    bound = egrad + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (grad.abs() + egrad) + 2.0 ** -126
    assert bool((off <= bound).all()), float((off / bound).max())


SIZES = [(1, 1, 1), (1, 2, 2), (3, 7, 7), (32, 10, 3), (5, 63, 5), (7, 64, 64), (6, 65, 1), (9, 255, 17), (4, 256, 256), (5, 1000, 10),
         (3, 1023, 300), (3, 1024, 1024), (3, 1025, 33), (2, 2047, 2), (33, 2048, 8), (2, 2049, 64), (3, 4095, 9), (2, 4097, 9),
         (2, 8191, 5), (3, 8200, 128), (2, 16385, 64), (5, 32000, 64), (3, 32003, 33), (2, 65536, 16), (2, 65537, 16), (1, 131080, 100),
         (2, 200001, 50), (600, 40, 4), (5000, 3, 2), (1300, 500, 6)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,k", SIZES)
def test_against_fp64(rows, classes, k, dtype):
    z, teacher, ids, labels = _inputs(dtype, rows, classes, k)
    st = _stage(dtype, rows, classes)
    for t, w in ((1.0, 0.0), (2.0, 0.5), (0.7, 0.25), (4.0, 1.0)):
        _compare(dtype, z, teacher, ids, labels, t, w, st=st)
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 40001])
def test_entries_absent_repeated_infinite(classes, dtype):
    import torch
    z, teacher, ids, labels = _inputs(dtype, 12, classes, 9)
    ids[1] = -1                                   # no entry at all
    ids[2, 3:] = -7                               # some
    ids[3, :] = classes - 1                       # one class nine times
    ids[4, 1], ids[4, 5] = ids[4, 0], ids[4, 0]   # three times among others
    teacher[5, 2:] = -np.inf                      # no probability
    teacher[6, :] = -np.inf                       # nor any
    teacher[7, :] = torch.finfo(torch.float32).min
    teacher[8, 4] = 80.0                          # all of it on one
    labels[9] = ids[9, 0]                         # label and entry on one class
    ids[10, 0], labels[10] = 0, 0
    for t, w in ((1.0, 0.0), (2.0, 0.5), (3.0, 1.0)):
        _compare(dtype, z, teacher, ids, labels, t, w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 40001, 140000])
def test_masked_classes_and_what_does_not_exist(classes, dtype):
    import torch
    z, teacher, ids, labels = _inputs(dtype, 6, classes, 4)
    st = _stage(dtype, 6, classes)
    # classes that the student cannot choose: -inf or the type's lowest value, neither among the entries nor the label
    free = torch.ones(6, classes, dtype=torch.bool, device="cuda")
    free.scatter_(1, ids.long(), False).scatter_(1, labels.long()[:, None], False)
    for low in (-np.inf, torch.finfo(z.dtype).min):
        masked = torch.where(free & (torch.arange(classes, device="cuda") % 3 == 0), low, z.float()).to(z.dtype)
        loss, grad = st.loss_distill(0, masked, teacher, ids, temperature=2.0, labels=labels, label_weight=0.5)
        want = _reference(torch.where(masked == low, -np.inf, masked.double()), teacher, ids, 2.0, labels, 0.5)
        _compare(dtype, torch.where(masked == low, -np.inf, masked.double()), teacher, ids, labels, 2.0, 0.5, got=(loss, grad))
        assert bool((grad[masked == low] == 0).all()) and want is not None
    # a class or label that does not exist: NaN, and the gradient of the other terms
    for change in ("id", "label"):
        i2, l2 = ids.clone(), labels.clone()
        if change == "id":
            i2[2, 1] = classes
        else:
            l2[3] = classes + 5
        loss, grad = st.loss_distill(0, z, teacher, i2, temperature=2.0, labels=l2, label_weight=0.5)
        assert np.isnan(float(loss))
        _, want, _, egrad = _reference(z, teacher, i2, 2.0, l2, 0.5)
        bound = egrad + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (want.abs() + egrad) + 2.0 ** -126
        assert bool(((grad.double() - want).abs() <= bound).all())
    # neither is read where its term has no weight
    loss, _ = st.loss_distill(0, z, teacher, torch.full_like(ids, -1), temperature=2.0, labels=labels, label_weight=1.0)
    assert np.isfinite(float(loss))
    loss, grad = st.loss_distill(0, z, teacher, ids, temperature=2.0, labels=None, label_weight=0.0)
    assert np.isfinite(float(loss))
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(5, 33), (3, 4100), (2, 140000), (3, 4096)])
def test_any_address_and_what_lies_around(rows, classes, dtype):
    import torch
    from paper_2509_23241_amd import binding as B
    z, teacher, ids, labels = _inputs(dtype, rows, classes, 5)
    st = _stage(dtype, rows, classes)
    for shift_in, shift_out in ((1, 1), (3, 0), (0, 5)):
        zin = torch.zeros(z.numel() + 32, dtype=z.dtype, device="cuda")
        zin[shift_in: shift_in + z.numel()] = z.reshape(-1)
        out = torch.full((z.numel() + 32,), 7.0, dtype=z.dtype, device="cuda")
        loss = torch.empty(1, device="cuda")
        es = z.element_size()
        B.stage_loss_distill(st.handle, 0, zin.data_ptr() + shift_in * es, teacher.data_ptr(), ids.data_ptr(), 5, 2.0, labels.data_ptr(), 0.5,
                             out.data_ptr() + shift_out * es, loss.data_ptr())
        _compare(dtype, z, teacher, ids, labels, 2.0, 0.5, got=(loss, out[shift_out: shift_out + z.numel()].view(z.shape)))
        assert bool((out[:shift_out] == 7.0).all()) and bool((out[shift_out + z.numel():] == 7.0).all())
    for refused in ((z.data_ptr(), z.data_ptr()), (z.data_ptr(), z.data_ptr() + es), (0, out.data_ptr())):
        with pytest.raises(B.StageLibError):
            B.stage_loss_distill(st.handle, 0, refused[0], teacher.data_ptr(), ids.data_ptr(), 5, 2.0, labels.data_ptr(), 0.5, refused[1],
                                 loss.data_ptr())
    with pytest.raises(B.StageLibError):          # weighted labels that are not there
        B.stage_loss_distill(st.handle, 0, z.data_ptr(), teacher.data_ptr(), ids.data_ptr(), 5, 2.0, 0, 0.5, out.data_ptr(), loss.data_ptr())
    st.close()


def test_token_positions_repeats_and_a_graph():
    """A row for every token position; calls repeat bit for bit, also from a captured graph on new logits."""
    import torch
    rows, tokens, classes, k = 3, 70, 777, 6
    st = _stage("bf16", rows, classes, tokens)
    z, teacher, ids, labels = _inputs("bf16", rows * tokens, classes, k)
    shaped = z.view(rows, tokens * classes)
    loss, grad = st.loss_distill(0, shaped, teacher, ids, temperature=2.0, labels=labels, label_weight=0.5)
    _compare("bf16", z, teacher, ids, labels, 2.0, 0.5, got=(loss, grad.view(z.shape)))
    for _ in range(3):
        again = st.loss_distill(0, shaped, teacher, ids, temperature=2.0, labels=labels, label_weight=0.5)
        assert torch.equal(loss, again[0]) and torch.equal(grad, again[1])
    st.close()
    stream = torch.cuda.Stream()
    from paper_2509_23241_amd.runner import GpuStage
    with torch.cuda.stream(stream):
        st = GpuStage([(8, classes, "none", tokens)], [np.zeros((classes, 8), np.float32), np.zeros(classes, np.float32)], dtype="bf16", mb=rows,
                      n=1, stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0, ring_capacity=1, max_in_flight=1,
                      stream=stream)
        st.forward(0, 0, torch.zeros(rows, 8 * tokens, dtype=torch.bfloat16, device="cuda"))
        held = shaped.clone()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = st.loss_distill(0, held, teacher, ids, temperature=2.0, labels=labels, label_weight=0.5)
        for seed in range(3):
            z2 = _inputs("bf16", rows * tokens, classes, k, seed=50 + seed)[0]
            held.copy_(z2.view(held.shape))
            graph.replay()
            stream.synchronize()
            _compare("bf16", z2, teacher, ids, labels, 2.0, 0.5, got=(out[0], out[1].view(z.shape)))
        st.close()


def test_a_student_learns_through_a_pipeline():
    """Windowed attention with its bias and the distillation loss in one training step of a two-stage pipeline, each stage on the
    oracle's formulas: outputs, loss and every gradient."""
    import torch
    from oracle import layers as L
    from oracle.stage import Stage
    from paper_2509_23241_amd.runner import GpuPipeline
    from parity_utils import TOL, oracle_flat_to_arena, rel_err, to_np
    from synth_inputs import workloads as W
    tokens, d, classes, k = 40, 32, 50, 5
    for dtype in ("f32", "bf16"):
        stages = (W.windowed_block(d, 4, 64, tokens, 2, 15, 2, 8, 30), W.windowed_block(d, 4, 64, tokens, 2, 15, 2, 8, 30) + (W.Dense(d, classes, "none", tokens=tokens),))
        w = W.Workload(name=f"student_{dtype}", dtype=dtype, stages=stages, mb=2, n=2, classes=classes)
        params = [W.init_params(w, s) for s in range(2)]
        rng = np.random.default_rng(1)
        x = w.cast(rng.standard_normal((4, tokens, d)))
        teacher = rng.standard_normal((4 * tokens, k)).astype(np.float32)
        ids = np.stack([rng.permutation(classes)[:k] for _ in range(4 * tokens)]).astype(np.int32)
        ids[::7, 2:] = -1
        labels = rng.integers(0, classes, 4 * tokens).astype(np.int32)
        storage = W.round_bf16 if dtype == "bf16" else None
        oracle = [Stage(s, p, policy="latest", lam=w.lam, lr=w.lr, momentum=w.momentum, n=2, first_stage=i == 0, storage=storage)
                  for i, (s, p) in enumerate(zip(stages, params))]
        mid = [oracle[0].forward(0, ub, x[2 * ub: 2 * ub + 2]) for ub in range(2)]
        logits = np.concatenate([oracle[1].forward(0, ub, mid[ub]) for ub in range(2)]).reshape(-1, classes)
        loss, dz = L.distill_loss(logits, teacher, ids, 2.0, labels, 0.25)
        dmid = oracle[1].backward(0, dz.reshape(4, tokens, classes) if storage is None else storage(dz.reshape(4, tokens, classes)))
        oracle[0].backward(0, dmid)
        pipe = GpuPipeline(w, params, policy="latest")
        seen = {}

        def on_event(what, ev, p, info):
            if what == "pre_update":
                seen[ev[2]] = to_np(p.stages[ev[2]].grad)

        given = dict(teacher=torch.from_numpy(teacher).cuda(), ids=torch.from_numpy(ids).cuda(), temperature=2.0, label_weight=0.25)
        tx = torch.from_numpy(x).to(pipe.stages[0].tdtype).cuda().reshape(4, -1)
        _, losses = pipe.run(1, lambda j: tx, lambda j: torch.from_numpy(labels).cuda(), on_event, get_teacher=lambda j: given)
        assert abs(float(losses[0]) - loss) <= TOL[dtype] * abs(loss)
        for s in range(2):
            want = oracle_flat_to_arena(pipe.stages[s], oracle[s].flat(oracle[s].g))
            err = rel_err(seen[s], want)
            print(dtype, s, err)
            assert err <= TOL[dtype]
        pipe.close()
