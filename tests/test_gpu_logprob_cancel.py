"""Policy losses whose rows nearly cancel, where every exponential is exact: what is left is how the rows' terms are formed and added up.

Logits are 0 or, hidden, -inf, so exponentials are 1 or 0, their sum is the number of classes that are left, and a log probability is minus
its logarithm.  Bound: the stored loss, 2^-24 of it; terms in fp64, for each a logarithm, an exponential of at most e^5 and some
operations, 32 roundings of 2^-53 to its parts, and as many for the sum over rows.  Rounded to fp32 the same terms miss it."""
import numpy as np
import pytest

from test_gpu_logprob import _stage

pytestmark = pytest.mark.gpu


def _case(classes, rows, kl, seed):
    """Logits, classes and the rest on the host; the exact terms and the size of their parts in fp64."""
    rng = np.random.default_rng(seed)
    z = np.zeros((rows, classes), np.float32)
    z[rng.random(z.shape) < rng.random((rows, 1)) * 0.8] = -np.inf
    ids = rng.integers(0, classes, rows).astype(np.int32)
    z[np.arange(rows), ids] = 0
    logp = -np.log((z == 0).sum(1).astype(np.float64))
    moved = rng.choice([-1.5, -0.4, -0.1, 0.05, 0.15, 0.5, 1.0], rows)
    old = (logp - moved).astype(np.float32)
    ref = (logp + rng.normal(size=rows)).astype(np.float32)
    adv = rng.normal(size=rows).astype(np.float32)
    weights = (rng.random(rows) + 0.5).astype(np.float32)

    def terms(adv):
        x = logp - old.astype(np.float64)
        ratio = np.exp(x)
        gain, inside = ratio * adv.astype(np.float64), np.clip(ratio, 0.8, 1.2) * adv.astype(np.float64)
        d = ref.astype(np.float64) - logp
        kl_term = kl * (np.expm1(d) - d)
        size = np.abs(np.minimum(gain, inside)) * (1 + np.abs(x)) + kl * (np.abs(np.expm1(d)) + np.abs(d)) * (1 + np.abs(d))
        return weights.astype(np.float64) * (kl_term - np.minimum(gain, inside)), weights * size
    # a row of ratio about one, in whose advantage the sum of the others is put
    old[0] = logp[0]
    for _ in range(4):
        t, _ = terms(adv)
        adv[0] += np.float32(t.sum() / weights[0])
    return z, ids, old, ref, adv, weights, *terms(adv)


@pytest.mark.parametrize("kl", [0.0, 0.1])
@pytest.mark.parametrize("classes,rows", [(10, 32), (50, 200), (100, 64), (1000, 40), (9000, 20), (70000, 12), (10, 20000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_nearly_cancel(classes, rows, dtype, kl):
    import torch
    z, ids, old, ref, adv, weights, terms, size = _case(classes, rows, kl, classes + rows)
    exact = float(np.sum(terms.astype(np.longdouble)))
    bound = 2.0 ** -24 * abs(exact) + (32 + rows) * 2.0 ** -53 * float(size.sum())
    rounded = float(np.sum(terms.astype(np.float32).astype(np.float64)))
    assert abs(rounded - exact) > 4 * bound, (rounded, exact, bound)     # the bound tells them apart
    st = _stage(dtype, rows, 1, classes)
    on = lambda v: torch.from_numpy(v).to("cuda")
    loss = st.loss_policy(0, on(z).to(st.tdtype), on(ids), on(old), on(adv), weights=on(weights), ref_logp=on(ref), kl_weight=kl)[0]
    print(float(loss), exact, "share of its bound", abs(float(loss) - exact) / bound)
    assert abs(float(loss) - exact) <= bound, (float(loss), exact, bound)
    st.close()
