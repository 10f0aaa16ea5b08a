"""Losses of so many rows that several workgroups add them up, rows on both sides of what a quarter of a wave, a wave and a workgroup hold, and
losses whose rows cancel; bounds as in test_gpu_logprob.py, where a probability is off by p of itself.

Of a class that is not the row's the gradient is slope times its probability q, so it is off by p of itself, too: its exponent, of at most
log2(e) spread, is rounded to 2^-24 of itself, which changes the power by ln 2 log2(e) spread f = spread f (11 f at a spread of 11, where 10 f are
allowed beside p q of it, next to nothing for a small q).  With hundreds of thousands of such classes that is met, and added here."""
import pytest

from test_gpu_logprob import U, _check, _logits, _policy_inputs, _policy_reference, _preference_reference, _row_parts, _stage

pytestmark = pytest.mark.gpu


def _with_powers(z, ids, want):
    """(loss, its bound, gradient, its bound, ..) with what is said above."""
    return want[:3] + (want[3] + _row_parts(z, ids)[3] * want[2].abs(),) + want[4:]



@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,tokens,classes", [(40001, 1, 20), (16384, 1, 3), (3, 5461, 9), (8200, 16, 40), (700, 100, 12)])
def test_policy_of_many_rows(seqs, tokens, classes, dtype):
    import torch
    z, ids, g = _logits(dtype, seqs, tokens, classes)
    old, adv, w, ref = _policy_inputs(z, ids, g, 0.2, 0.2)
    st = _stage(dtype, seqs, tokens, classes)
    want = _with_powers(z, ids, _policy_reference(z, ids, old, adv, None, ref, 0.2, 0.2, 0.1, U[dtype]))
    first = st.loss_policy(0, z, ids, old, adv, ref_logp=ref, kl_weight=0.1)
    _check("policy", first, *want)
    for _ in range(3):
        for a, b in zip(first, st.loss_policy(0, z, ids, old, adv, ref_logp=ref, kl_weight=0.1)):
            assert torch.equal(a, b)
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,tokens,classes", [(40002, 1, 12), (33000, 2, 20), (4, 5000, 30), (2, 4097, 17)])
def test_preference_of_many_rows(seqs, tokens, classes, dtype):
    import torch
    z, ids, g = _logits(dtype, seqs, tokens, classes)
    w = torch.rand(z.shape[0], generator=g, device="cuda")
    logp = _row_parts(z, ids)[1]
    ref = ((torch.where(ids >= 0, w, 0.0) * logp).view(seqs, tokens).sum(1) + torch.randn(seqs, generator=g, device="cuda")).float()
    st = _stage(dtype, seqs, tokens, classes)
    want = _with_powers(z, ids, _preference_reference(z, ids, w, ref, tokens, 0.3, 0.1, U[dtype]))
    first = st.loss_preference(0, z, ids, ref, weights=w, beta=0.3, label_smoothing=0.1)
    _check("preference", first, *want)
    for _ in range(3):
        for a, b in zip(first, st.loss_preference(0, z, ids, ref, weights=w, beta=0.3, label_smoothing=0.1)):
            assert torch.equal(a, b)
    st.close()


@pytest.mark.parametrize("dtype,V", [("f32", 4), ("bf16", 8)])
@pytest.mark.parametrize("units", [16, 32, 64, 128, 256, 512, 1024])
def test_rows_at_the_borders(units, dtype, V):
    """classes / V + 2 units on either side of a border, rows that start anywhere within 16 bytes where their number is odd."""
    import torch
    for classes in ((units - 2) * V + V - 1, (units - 1) * V, (units - 1) * V + 1):
        z, ids, g = _logits(dtype, 10, 5, classes)
        old, adv, w, ref = _policy_inputs(z, ids, g, 0.2, 0.2)
        st = _stage(dtype, 10, 5, classes)
        want = _with_powers(z, ids, _policy_reference(z, ids, old, adv, w, ref, 0.2, 0.2, 0.1, U[dtype]))
        got = st.loss_policy(0, z, ids, old, adv, weights=w, ref_logp=ref, kl_weight=0.1)
        gone = (ids < 0) | (w == 0)
        _check(classes, (got[0], got[1], torch.where(gone, 0.0, got[2])), *want[:4], torch.where(gone, 0.0, want[4]), want[5])
        pair_ref = torch.zeros(10, device="cuda")
        _check(classes, st.loss_preference(0, z, ids, pair_ref), *_with_powers(z, ids, _preference_reference(z, ids, None, pair_ref, 5, 0.1, 0.0, U[dtype])))
        st.close()


def test_rows_that_cancel():
    """Ratios of one, every advantage with its opposite on an equal row: the sum is 0 to fp64's rounding of terms of order one."""
    import torch
    z, ids, g = _logits("f32", 32, 1, 10)
    z[16:], ids[16:] = z[:16], ids[:16].clamp(min=0)
    ids[:16] = ids[16:]
    adv = torch.randn(32, generator=g, device="cuda")
    adv[16:] = -adv[:16]
    logp = _row_parts(z, ids)[1].float()
    st = _stage("f32", 32, 1, 10)
    loss = st.loss_policy(0, z, ids, logp, adv)[0]
    assert abs(float(loss)) <= 32 * 2.0 ** -52 * float(adv.abs().max()), float(loss)
    st.close()
