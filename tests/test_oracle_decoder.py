"""The oracle's gated layer, rotary positions and losses on log probabilities: gradients against central differences in fp64, and
properties that hold whatever the numbers."""
import numpy as np
import pytest

from oracle import layers as L
from synth_inputs import workloads as W

STEP = 1e-6   # central differences of smooth functions of order one: their own error is of order STEP^2 and 1e-16 / STEP


def _difference(f, x, direction):
    return (f(x + STEP * direction) - f(x - STEP * direction)) / (2 * STEP)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu", "none"])
def test_gated_gradient(act):
    rng = np.random.default_rng(1)
    x, w, b, dy = (rng.standard_normal(s) for s in ((2, 5, 7), (12, 7), (12,), (2, 5, 6)))
    dz = L.gated_backward(dy, L.dense_forward(x, w, b), act)
    dw, db, dx = L.dense_backward(dz, x, w)
    loss = lambda x, w, b: (L.gated_forward(L.dense_forward(x, w, b), act) * dy).sum()
    for grad, at, f in ((dx, x, lambda v: loss(v, w, b)), (dw, w, lambda v: loss(x, v, b)), (db, b, lambda v: loss(x, w, v))):
        u = rng.standard_normal(at.shape)
        assert abs(_difference(f, at, u) - (grad * u).sum()) < 1e-7 * (1 + abs((grad * u).sum()))


@pytest.mark.parametrize("spec", [W.Rotary(3, 1, 8, 6, 8), W.Rotary(2, 2, 7, 5, 4, "pairs", first=3), W.Rotary(4, 2, 6, 9, 6, factor=4.0),
                                  W.Rotary(1, 1, 16, 9, 16, "pairs", 100.0, 0, 8.0, 20, 0.5, 2.0, 1.25)], ids=str)
def test_rotary(spec):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 2, spec.tokens, (spec.heads + 2 * spec.kv_heads) * spec.head))
    y = L.rotary(x, spec)
    # linear, so its gradient is the transpose: <turn x, dy> = <x, turn back dy>
    assert abs((y * dy).sum() - (x * L.rotary(dy, spec, back=True)).sum()) < 1e-12 * np.abs(x).sum()
    heads = (spec.heads + spec.kv_heads) * spec.head
    assert np.array_equal(y[..., heads:], x[..., heads:])                       # values pass
    parts, turned = (v[..., :heads].reshape(2, spec.tokens, -1, spec.head) for v in (x, y))
    assert np.array_equal(turned[..., spec.rotated:], parts[..., spec.rotated:])
    assert np.allclose(np.linalg.norm(turned[..., :spec.rotated], axis=-1), spec.amplitude * np.linalg.norm(parts[..., :spec.rotated], axis=-1))
    if spec.first == 0:
        assert np.allclose(y[:, 0, :heads].reshape(-1, spec.head)[:, :spec.rotated],
                           spec.amplitude * x[:, 0, :heads].reshape(-1, spec.head)[:, :spec.rotated])


def test_rotary_layouts_are_permutations_of_each_other():
    rng = np.random.default_rng(3)
    halves, pairs = W.Rotary(2, 1, 12, 7, 8, "halves"), W.Rotary(2, 1, 12, 7, 8, "pairs")
    x = rng.standard_normal((1, 7, 4, 12))
    order = np.concatenate([np.arange(8).reshape(2, 4).T.reshape(-1), np.arange(8, 12)])     # (i, i + 4) side by side
    a = L.rotary(x.reshape(1, 7, 48), halves).reshape(1, 7, 4, 12)[..., order]
    b = L.rotary(x[..., order].reshape(1, 7, 48), pairs).reshape(1, 7, 4, 12)
    b[:, :, 3] = a[:, :, 3]                                                                   # values: permuted, not turned
    assert np.allclose(a, b)


def test_rotary_speeds_by_parts():
    """Fast pairs as they are, slow ones slowed down by the factor, a ramp between."""
    spec = W.Rotary(1, 1, 64, 4, 64, factor=8.0, original=1024, low=1.0, high=4.0)
    plain = L.rotary_speeds(W.Rotary(1, 1, 64, 4, 64))
    speeds, turns = L.rotary_speeds(spec), 1024 * plain / (2 * np.pi)
    assert np.allclose(speeds[turns >= 4], plain[turns >= 4]) and np.allclose(speeds[turns <= 1], plain[turns <= 1] / 8)
    ramp = (turns > 1) & (turns < 4)
    assert ramp.any() and ((speeds < plain) & (speeds > plain / 8))[ramp].all() and (np.diff(speeds) < 0).all()


def test_library_speeds_are_the_oracles():
    """Through the description: float32 fields, the same formula (the library's is host code; this pins what they are made of)."""
    from paper_2509_23241_amd import binding as B
    d = B.make_desc([("rotary", 4, 2, 64, 8, 32, "pairs", 500000.0, 7, 8.0, 8192, 1.0, 4.0, 1.25)], dtype="f32", mb=1, n=1, stage_index=0,
                    num_stages=1, ring_capacity=1, max_in_flight=1, policy="latest", needs_dx=True, lam=0.1, lr=0.0, momentum=0.0)
    l = d.layers[0]
    assert list(l.geom) == [8, 4, 2, 32, 0] and list(l.rel) == [7, 8192] and list(l.rope) == [500000.0, 8.0, 1.0, 4.0, 1.25]
    assert l.in_features == l.out_features == 8 * 64


@pytest.mark.parametrize("kind", ["policy", "policy_kl", "preference", "preference_smooth"])
def test_loss_gradients(kind):
    rng = np.random.default_rng(4)
    rows, classes, tokens = 24, 9, 3
    z = rng.standard_normal((rows, classes))
    ids = rng.integers(0, classes, rows)
    ids[::5] = -1
    w = rng.uniform(0, 1, rows)
    logp = np.log(np.exp(z) / np.exp(z).sum(1, keepdims=True))[np.arange(rows), ids]
    if kind.startswith("policy"):
        old, adv, ref = logp - 0.3 * rng.standard_normal(rows), rng.standard_normal(rows), logp + rng.standard_normal(rows)
        f = lambda v: L.policy_loss(v, ids, old, adv, w, ref, 0.2, 0.3, 0.5 if kind == "policy_kl" else 0.0)
    else:
        f = lambda v: L.preference_loss(v, ids, rng2, tokens, w, 0.7, 0.2 if kind.endswith("smooth") else 0.0)
        rng2 = rng.standard_normal(rows // tokens)
    u = rng.standard_normal(z.shape)
    want = (f(z)[1] * u).sum()
    assert abs(_difference(lambda v: f(v)[0], z, u) - want) < 1e-6 * (1 + abs(want))
    assert (f(z)[1][ids < 0] == 0).all() and (f(z)[2][ids < 0] == 0).all()
    assert np.abs(f(z)[1].sum(1)).max() < 1e-12                       # adding a constant to a row's logits changes nothing


def test_losses_at_known_points():
    z = np.zeros((4, 5))
    loss, dz, logp = L.policy_loss(z, np.array([0, 1, 2, 3]), np.full(4, -np.log(5)), np.array([1.0, -1.0, 2.0, 0.0]))
    assert abs(loss + 0.5) < 1e-12 and np.allclose(logp, -np.log(5))  # ratios of one: minus the mean advantage
    loss, dz, logp = L.preference_loss(z, np.array([0, 1, 2, 3]), np.zeros(2), 2)
    assert abs(loss - np.log(2)) < 1e-12                              # no preference either way
    assert np.allclose(dz[:2].sum(0) + dz[2:].sum(0), 0.05 / 1 * np.array([-1, -1, 1, 1, 0]))
