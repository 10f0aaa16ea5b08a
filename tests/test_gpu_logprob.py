"""Log probabilities of given classes, the clipped policy loss and the preference loss (kernels_logprob.hip), with their gradients,
against fp64: sizes around what a workgroup holds, rows without a term, masked classes, ratios on both sides of the clip, alignment.

Bounds, f = 2^-24, u = f in fp32 and 2^-8 in bf16: an exponent has an error of 4 f (spread + 1) (the scale, the product, the difference), a
sum of n terms over lanes (n / 64 + 32) f; so probabilities are off by p = (4 (spread + 1) + classes / 64 + 32) f of themselves,
log probabilities by p + f |l| (stored).  A ratio is off by p + 4 f (1 + |l - o|) of itself, exp(d) likewise; a row's slope (what its
loss changes by with l) by the sum of what its terms are; a gradient by slope times 8 f + p, what the slope is off, and u.  Sequence
sums are formed in fp64 of stored l: their error is the sum of theirs; sigmoids change by at most a quarter of what their argument is off."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
F = 2.0 ** -24
U = {"f32": F, "bf16": 2.0 ** -8}


def _stage(dtype, seqs, tokens, classes, n=1):
    import torch
    from paper_2509_23241_amd.runner import GpuStage
    st = GpuStage([(8, classes, "none", tokens)], [np.zeros((classes, 8), np.float32), np.zeros(classes, np.float32)], dtype=dtype,
                  mb=seqs // n, n=n, stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0, ring_capacity=1, max_in_flight=1)
    for ub in range(n):
        st.forward(0, ub, torch.zeros(seqs // n, 8 * tokens, dtype=st.tdtype, device="cuda"))
    return st


def _logits(dtype, seqs, tokens, classes, seed=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + seqs + 11 * tokens + classes)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows = seqs * tokens
    z = (3 * torch.randn(rows, classes, generator=g, device="cuda")).to(t)
    ids = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    ids[3::7] = -1
    ids[5::14] = -100
    return z, ids, g


def _row_parts(z, ids):
    """softmax, log probability (0 without a class), one-hot, relative error of a probability, absolute error of a log probability."""
    import torch
    rows, classes = z.shape
    z = z.double()
    there = (ids >= 0) & (ids < classes)
    at = ids.long().clamp(0, classes - 1)[:, None]
    logs = z.log_softmax(1)
    logp = torch.where(there, logs.gather(1, at)[:, 0], 0.0)
    one = torch.zeros_like(z).scatter_(1, at, there.double()[:, None])
    finite = z.masked_fill(~torch.isfinite(z), 0)
    p = (4 * (float((finite.max() - finite.min()).abs()) + 1) + classes / 64 + 32) * F
    return logs.exp(), logp, one, p, there * (p + F * logp.abs())


def _policy_reference(z, ids, old, adv, w, ref, low, high, kl, u):
    import torch
    soft, logp, one, p, elogp = _row_parts(z, ids)
    there = (ids >= 0) & (ids < z.shape[1])
    w = torch.full_like(old, 1 / z.shape[0]) if w is None else w
    w, adv = (torch.where(there, v.double(), 0.0) for v in (w, adv))
    moved = torch.where(there, logp - old.double(), 0.0)
    ratio = moved.exp()
    gain, inside = ratio * adv, ratio.clamp(1 - low, 1 + high) * adv
    value, slope = -torch.minimum(gain, inside), torch.where(gain <= inside, -gain, 0.0)
    eslope = slope.abs() * (p + 4 * F * (1 + moved.abs()))
    evalue = eslope + 4 * F * value.abs()
    if kl > 0:
        d = torch.where(there, ref.double() - logp, 0.0)
        value = value + kl * (torch.expm1(d) - d)
        slope = slope - kl * torch.expm1(d)
        eslope = eslope + kl * (d.exp() * (p + 4 * F * (1 + d.abs())) + 4 * F * torch.expm1(d).abs())
        evalue = evalue + kl * (torch.expm1(d).abs() * elogp + 4 * F * d.abs() * d.exp() + 8 * F * (torch.expm1(d).abs() + d.abs()))
    grad, egrad = _gradient(soft, one, w * slope, w.abs() * (eslope + 2 * F * slope.abs()), p, u)
    return (w * value).sum(), (w.abs() * (evalue + 2 * F * value.abs())).sum(), grad, egrad, logp, elogp


def _gradient(soft, one, slope, eslope, p, u):
    slope, eslope = slope[:, None], eslope[:, None]
    grad = slope * (one - soft)
    return grad, (slope.abs() * (8 * F + p * soft + 2 * F) + eslope) * (one + soft) + u * grad.abs() * (1 + u) + 2.0 ** -126


def _preference_reference(z, ids, w, ref, tokens, beta, smooth, u):
    import torch
    soft, logp, one, p, elogp = _row_parts(z, ids)
    w = torch.where(ids >= 0, torch.ones_like(logp) if w is None else w.double(), 0.0)
    each = lambda v: v.view(-1, 2, tokens).sum(2)
    s = each(w * logp) - ref.double().view(-1, 2)
    m = beta * (s[:, 0] - s[:, 1])
    em = beta * each(w.abs() * elogp).sum(1)
    sig, log_sig = torch.sigmoid, torch.nn.functional.logsigmoid
    loss = -((1 - smooth) * log_sig(m) + smooth * log_sig(-m))
    pairs = m.numel()
    pull = beta / pairs * (smooth * sig(m) - (1 - smooth) * sig(-m))
    epull = beta / pairs * em / 4 + F * pull.abs()
    rows = lambda v, sign: torch.stack([v, sign * v], 1).view(-1, 1).expand(-1, tokens).reshape(-1) * (w if sign < 0 else w.abs())
    grad, egrad = _gradient(soft, one, rows(pull, -1), rows(epull, 1) + 2 * F * rows(pull, -1).abs(), p, u)
    return loss.mean(), (em + 2 * F * loss).mean(), grad, egrad, logp, elogp


def _check(name, got, loss, eloss, grad, egrad, logp, elogp):
    import torch
    assert abs(float(got[0]) - float(loss)) <= float(eloss) + F * abs(float(loss)), (name, float(got[0]), float(loss), float(eloss))
    over = float(((got[1].double().view(grad.shape) - grad).abs() / egrad).max())
    assert over <= 1.0, (name, "gradient", over)
    _check_logp(name, got[2], logp, elogp)


def _check_logp(name, got, logp, elogp):
    over = float(((got.double() - logp).abs() / (elogp + 1e-30)).max())
    assert over <= 1.0, (name, "log probability", over)


def _policy_inputs(z, ids, g, low, high):
    """Old log probabilities on both sides of the clip borders, not within 1e-3 of them."""
    import torch
    logp = _row_parts(z, ids)[1]
    rows = z.shape[0]
    normal = lambda: torch.randn(rows, generator=g, device="cuda")
    moved = 0.3 * normal().double()
    for border in (np.log1p(-low) if low < 1 else -np.inf, np.log1p(high)):
        moved += torch.where((moved - border).abs() < 1e-3, 4e-3, 0.0)
    adv = normal()
    adv[::9] = 0
    w = torch.rand(rows, generator=g, device="cuda") / rows
    w[::5] = 0
    return (logp - moved).float(), adv, w, (logp + 0.4 * normal()).float()


SIZES = [(1, 1, 1), (1, 2, 2), (3, 1, 7), (32, 1, 10), (2, 9, 63), (7, 1, 64), (6, 2, 65), (3, 3, 255), (4, 1, 256), (5, 4, 1000), (1, 3, 1023),
         (1, 3, 1024), (3, 1, 1025), (2, 1, 2047), (33, 2, 2048), (2, 1, 2049), (3, 1, 4095), (2, 2, 4097), (2, 1, 8191), (3, 1, 8200),
         (2, 1, 16385), (5, 3, 32000), (3, 1, 32003), (2, 1, 65536), (2, 1, 65537), (1, 1, 131080), (2, 1, 200001), (300, 2, 40), (5000, 1, 3),
         (13, 100, 500)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,tokens,classes", SIZES)
def test_log_probabilities_and_policy_against_fp64(seqs, tokens, classes, dtype):
    import torch
    z, ids, g = _logits(dtype, seqs, tokens, classes)
    st = _stage(dtype, seqs, tokens, classes)
    _, logp, _, _, elogp = _row_parts(z, ids)
    _check_logp("logprobs", st.logprobs(z, ids), logp, elogp)
    part = max(1, z.shape[0] // 2)
    _check_logp("some rows", st.logprobs(z[:part], ids[:part]), logp[:part], elogp[:part])
    for low, high, kl, weighted in ((0.2, 0.2, 0.0, False), (0.2, 0.28, 0.05, True), (1.0, 3.0, 1.0, False), (0.0, 0.0, 0.5, True)):
        old, adv, w, ref = _policy_inputs(z, ids, g, low, high)
        w = w if weighted else None
        want = _policy_reference(z, ids, old, adv, w, ref, low, high, kl, U[dtype])
        got = st.loss_policy(0, z, ids, old, adv, weights=w, ref_logp=ref if kl else None, clip_low=low, clip_high=high, kl_weight=kl)
        gone = (ids < 0) | (torch.zeros_like(adv) if w is None else (w == 0).float()).bool()
        _check((low, high, kl), (got[0], got[1], torch.where(gone, 0.0, got[2])), *want[:4], torch.where(gone, 0.0, want[4]), want[5])
        assert bool((got[1].view(z.shape)[gone] == 0).all()) and bool((got[2][gone] == 0).all())
    st.close()


PAIRS = [(2, 1, 1), (2, 1, 2), (4, 3, 7), (2, 64, 10), (6, 5, 65), (2, 300, 33), (64, 2, 100), (2, 7, 1000), (4, 3, 2049), (2, 2, 8200),
         (2, 5, 32000), (6, 1, 32003), (2, 2, 65537), (2, 1, 200001), (600, 1, 12), (10, 70, 520)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,tokens,classes", PAIRS)
def test_preference_against_fp64(seqs, tokens, classes, dtype):
    import torch
    z, ids, g = _logits(dtype, seqs, tokens, classes)
    w = torch.rand(z.shape[0], generator=g, device="cuda")
    w[1::4] = 0
    logp = _row_parts(z, ids)[1]
    st = _stage(dtype, seqs, tokens, classes)
    for beta, smooth, weights in ((0.1, 0.0, None), (0.5, 0.1, w), (2.0, 1.0, w), (0.0, 0.5, None)):
        eff = torch.where(ids >= 0, torch.ones_like(w) if weights is None else weights, 0.0)
        ref = ((eff * logp).view(seqs, tokens).sum(1) + 5 * torch.randn(seqs, generator=g, device="cuda")).float()
        got = st.loss_preference(0, z, ids, ref, weights=weights, beta=beta, label_smoothing=smooth)
        want = _preference_reference(z, ids, weights, ref, tokens, beta, smooth, U[dtype])
        gone = eff == 0
        _check((beta, smooth), (got[0], got[1], got[2]), *want[:4], torch.where(gone, 0.0, want[4]), want[5])
        assert bool((got[1].view(z.shape)[gone] == 0).all()) and bool((got[2][gone] == 0).all())
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 40001, 140000])
def test_masked_classes(classes, dtype):
    """Classes that cannot be chosen, -inf or the type's lowest value: no probability, no gradient."""
    import torch
    z, ids, g = _logits(dtype, 4, 2, classes)
    st = _stage(dtype, 4, 2, classes)
    free = torch.ones_like(z, dtype=torch.bool).scatter_(1, ids.long().clamp(min=0)[:, None], False)
    hide = free & (torch.arange(classes, device="cuda") % 3 == 0)
    old, adv, w, ref = _policy_inputs(z, ids, g, 0.2, 0.2)
    pair_ref = torch.zeros(4, device="cuda")
    for low in (-np.inf, torch.finfo(z.dtype).min):
        masked = torch.where(hide, low, z.float()).to(z.dtype)
        exact = torch.where(hide, -np.inf, z.double())
        want = _policy_reference(exact, ids, old, adv, None, ref, 0.2, 0.2, 0.1, U[dtype])
        got = st.loss_policy(0, masked, ids, old, adv, ref_logp=ref, kl_weight=0.1)
        _check("policy", got, *want)
        assert bool((got[1].view(z.shape)[hide] == 0).all())
        want = _preference_reference(exact, ids, None, pair_ref, 2, 0.1, 0.2, U[dtype])
        got = st.loss_preference(0, masked, ids, pair_ref, label_smoothing=0.2)
        _check("preference", got, *want)
        assert bool((got[1].view(z.shape)[hide] == 0).all())
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 40001, 140000])
def test_rows_without_a_term_may_hold_anything(classes, dtype):
    """Padding: NaN and infinities in its logits, ratios and advantages reach nothing."""
    import torch
    z, ids, g = _logits(dtype, 6, 3, classes)
    st = _stage(dtype, 6, 3, classes)
    old, adv, w, ref = _policy_inputs(z, ids, g, 0.2, 0.2)
    gone = (ids < 0) | (w == 0)
    nan = float("nan")
    dirty = z.clone()
    dirty[gone] = nan
    dirty[gone, ::2] = float("inf")
    spoil = lambda v: torch.where(gone, nan, v)
    clean = st.loss_policy(0, z, ids, old, adv, weights=w, ref_logp=ref, kl_weight=0.1)
    got = st.loss_policy(0, dirty, ids, spoil(old), spoil(adv), weights=w, ref_logp=spoil(ref), kl_weight=0.1)
    for a, b in zip(clean, got):
        assert torch.equal(a, b)
    pair_ref = torch.zeros(6, device="cuda")
    clean = st.loss_preference(0, z, ids, pair_ref, weights=w)
    got = st.loss_preference(0, dirty, ids, pair_ref, weights=w)
    for a, b in zip(clean, got):
        assert torch.equal(a, b)
    none = torch.full_like(ids, -1)                       # not a row left: losses of nothing
    loss, grad, logp = st.loss_policy(0, dirty, none, spoil(old), spoil(adv), weights=w)
    assert float(loss) == 0 and bool((grad == 0).all()) and bool((logp == 0).all())
    loss, grad, logp = st.loss_preference(0, dirty, none, pair_ref)
    assert abs(float(loss) - np.log(2)) <= 2 * F and bool((grad == 0).all()) and bool((logp == 0).all())
    assert bool((st.logprobs(dirty, none) == 0).all())
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 40001, 140000])
def test_a_class_that_does_not_exist(classes, dtype):
    import torch
    z, ids, g = _logits(dtype, 4, 3, classes)
    st = _stage(dtype, 4, 3, classes)
    old, adv, w, ref = _policy_inputs(z, ids, g, 0.2, 0.2)
    bad = ids.clone()
    bad[7] = classes
    others = torch.arange(12, device="cuda") != 7
    clean, got = st.loss_policy(0, z, ids, old, adv), st.loss_policy(0, z, bad, old, adv)
    assert bool(torch.isnan(got[0]).all()) and bool(torch.isnan(got[2][7]))
    assert torch.equal(got[1].view(z.shape)[others], clean[1].view(z.shape)[others]) and bool((got[1].view(z.shape)[7] == 0).all())
    assert torch.equal(got[2][others], clean[2][others])
    pair_ref = torch.zeros(4, device="cuda")
    clean, got = st.loss_preference(0, z, ids, pair_ref), st.loss_preference(0, z, bad, pair_ref)
    assert bool(torch.isnan(got[0]).all())
    assert torch.equal(got[1].view(z.shape)[:6], clean[1].view(z.shape)[:6])   # rows of the other pair
    counted = bad >= 0
    assert bool(torch.isnan(got[1].view(z.shape)[6:][counted[6:]].float()).all())
    assert bool(torch.isnan(st.logprobs(z, bad)[7])) and torch.equal(st.logprobs(z, bad)[others], st.logprobs(z, ids)[others])
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [12, 1000, 33000])
def test_large_logits(classes, dtype):
    """Logits around 1000, 1e5 and 1e9: what the maximum is rounded by takes no part.  The bound grows with the spread alone."""
    import torch
    z, ids, g = _logits("f32", 4, 2, classes)
    st = _stage(dtype, 4, 2, classes)
    for at in (1000.0, -1e5, 1e9, 3e38):
        moved = (z + at).to(st.tdtype)
        _, logp, _, p, elogp = _row_parts(moved, ids)
        _check_logp(at, st.logprobs(moved, ids), logp, elogp)
        old, adv, w, ref = _policy_inputs(moved, ids, g, 0.2, 0.2)
        _check(at, st.loss_policy(0, moved, ids, old, adv, ref_logp=ref, kl_weight=0.1),
               *_policy_reference(moved, ids, old, adv, None, ref, 0.2, 0.2, 0.1, U[dtype]))
    st.close()


def test_far_ratios():
    """Ratios of e^80 and e^-80 either way, zero advantages beside infinite ratios, references far off."""
    import torch
    z, ids, g = _logits("f32", 12, 1, 50)
    ids = ids.clamp(min=0)
    st = _stage("f32", 12, 1, 50)
    logp = _row_parts(z, ids)[1]
    moved = torch.tensor([80.0, -80.0, 80.0, -80.0, 0.0, 2.0, -2.0, 500.0, -500.0, 0.5, -0.5, 500.0], device="cuda").double()
    adv = torch.tensor([1.0, 1.0, -1.0, -1.0, 3.0, -2.0, 2.0, 0.0, 1.0, 1.0, -1.0, 2.0], device="cuda")
    old = (logp - moved).float()
    _check("far", st.loss_policy(0, z, ids, old, adv), *_policy_reference(z, ids, old, adv, None, None, 0.2, 0.2, 0.0, F))
    ref = (logp + torch.linspace(-60, 40, 12, device="cuda").double()).float()
    _check("reference", st.loss_policy(0, z, ids, logp.float(), adv, ref_logp=ref, kl_weight=0.01),
           *_policy_reference(z, ids, logp.float(), adv, None, ref, 0.2, 0.2, 0.01, F))
    pair_ref = torch.tensor([0.0, 2000.0, 2000.0, 0.0] * 3, device="cuda")   # margins of hundreds either way
    got = st.loss_preference(0, z, ids, pair_ref, beta=1.0)
    _check("margins", got, *_preference_reference(z, ids, None, pair_ref, 1, 1.0, 0.0, F))
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [65, 2049, 32003])
def test_logits_and_gradients_at_odd_addresses(classes, dtype):
    import torch
    z, ids, g = _logits(dtype, 4, 2, classes)
    st = _stage(dtype, 4, 2, classes)
    from paper_2509_23241_amd import binding as B
    old, adv, w, ref = _policy_inputs(z, ids, g, 0.2, 0.2)
    want = _policy_reference(z, ids, old, adv, w, ref, 0.2, 0.2, 0.1, U[dtype])
    gone = (ids < 0) | (w == 0)
    pair_ref = torch.zeros(4, device="cuda")
    pair = _preference_reference(z, ids, None, pair_ref, 2, 0.1, 0.0, U[dtype])
    for here, there in ((1, 1), (1, 3), (0, 2), (5, 5)):
        at = lambda k: torch.zeros(z.numel() + 16, dtype=z.dtype, device="cuda")[k: k + z.numel()]
        zz, grad = at(here).copy_(z.view(-1)), at(there)
        loss, logp = torch.empty(1, device="cuda"), torch.empty(8, device="cuda")
        B.stage_loss_policy(st.handle, 0, zz.data_ptr(), ids.data_ptr(), old.data_ptr(), adv.data_ptr(), w.data_ptr(), ref.data_ptr(), 0.2, 0.2,
                            0.1, grad.data_ptr(), logp.data_ptr(), loss.data_ptr())
        _check((here, there), (loss, grad, torch.where(gone, 0.0, logp)), *want[:4], torch.where(gone, 0.0, want[4]), want[5])
        B.stage_loss_preference(st.handle, 0, zz.data_ptr(), ids.data_ptr(), 0, pair_ref.data_ptr(), 0.1, 0.0, grad.data_ptr(), logp.data_ptr(),
                                loss.data_ptr())
        _check((here, there), (loss, grad, logp), *pair)
        _check_logp((here, there), st.logprobs(zz, ids), _row_parts(z, ids)[1], _row_parts(z, ids)[4])
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeated_calls_and_many_rows_give_the_same_bits(dtype):
    """A row's results do not depend on how many others there are, nor on what ran before."""
    import torch
    z, ids, g = _logits(dtype, 6, 50, 700)
    old, adv, w, ref = _policy_inputs(z, ids, g, 0.2, 0.2)
    st = _stage(dtype, 6, 50, 700)
    a = st.loss_policy(0, z, ids, old, adv, weights=w, ref_logp=ref, kl_weight=0.1)
    pair_ref = torch.zeros(6, device="cuda")
    b = st.loss_preference(0, z, ids, pair_ref)
    for _ in range(3):
        for x, y in zip(a + b, st.loss_policy(0, z, ids, old, adv, weights=w, ref_logp=ref, kl_weight=0.1) + st.loss_preference(0, z, ids, pair_ref)):
            assert torch.equal(x, y)
    st.close()
    st = _stage(dtype, 1, 50, 700)
    one = st.loss_policy(0, z[:50], ids[:50], old[:50], adv[:50], weights=w[:50], ref_logp=ref[:50], kl_weight=0.1)
    assert torch.equal(one[1].view(50, -1), a[1].view(300, -1)[:50]) and torch.equal(one[2], a[2][:50])
    st.close()


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_gradients_against_differences(kind):
    """What the loss changes by over a step of the logits either way, against the gradient times the step (fp32).  Allowed: what both losses
    and the gradient are off by their bounds, and the step's own curvature in fp64."""
    import torch
    z, ids, g = _logits("f32", 4, 5, 30)
    old, adv, w, ref = _policy_inputs(z, ids, g, 0.2, 0.2)
    old = (_row_parts(z, ids)[1] + 0.05).float()           # ratios that stay inside the borders
    pair_ref = torch.zeros(4, device="cuda")
    st = _stage("f32", 4, 5, 30)
    if kind == "policy":
        run = lambda v: st.loss_policy(0, v, ids, old, adv, weights=w, ref_logp=ref, kl_weight=0.3)
        exact = lambda v: _policy_reference(v, ids, old, adv, w, ref, 0.2, 0.2, 0.3, F)
    else:
        run = lambda v: st.loss_preference(0, v, ids, pair_ref, weights=20 * w, beta=0.3, label_smoothing=0.1)
        exact = lambda v: _preference_reference(v, ids, 20 * w, pair_ref, 5, 0.3, 0.1, F)
    direction = torch.randn(z.shape, generator=g, device="cuda") * 0.02
    sides = [z + direction, z - direction]
    step = (sides[0] - sides[1]).double()
    change = float(run(sides[0])[0].double() - run(sides[1])[0].double())
    refs = [exact(v) for v in sides]
    mid = exact(z)
    allowed = sum(float(r[1] + F * r[0].abs()) for r in refs) + float((mid[3] * step.abs()).sum())
    curved = abs(float(refs[0][0] - refs[1][0]) - float((mid[2] * step).sum()))
    got = float((run(z)[1].double() * step).sum())
    assert abs(change - got) <= allowed + curved, (change, got, allowed, curved)
    assert allowed + curved < 0.2 * abs(got)
    st.close()
