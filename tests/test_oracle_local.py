"""Pins of the oracle's windowed attention, distance buckets and distillation loss: index loops, closed forms, finite differences."""
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import layers as L
from oracle.stage import Stage
from synth_inputs import workloads as W


@pytest.mark.parametrize("buckets,reach", [(2, 2), (4, 64), (5, 3), (5, 1024), (32, 128), (32, 512), (64, 64), (128, 65), (128, 4096)])
def test_first_distances_are_the_smallest_whole_ones(buckets, reach):
    first = L.first_distances(buckets, reach)
    half, n = buckets // 2, buckets - buckets // 2
    assert first[:half + 1] == list(range(half + 1))
    assert len(first) == buckets and all(a <= b for a, b in zip(first, first[1:])) and first[-1] <= reach
    for t in range(n):
        at, ratio = first[half + t], Fraction(reach, half)
        assert Fraction(at, half) ** n >= ratio ** t                       # not below its border
        assert at == half or Fraction(at - 1, half) ** n < ratio ** t      # and the one before it is
    bucket = L.distance_buckets(reach + 5, buckets, reach)
    assert bucket[0] == 0 and bucket[reach] == buckets - 1 and bucket[-1] == buckets - 1
    for b in range(buckets):
        for d in np.flatnonzero(bucket == b):
            assert first[b] <= d and (b == buckets - 1 or d < first[b + 1])


def _loops(x, spec, table):
    B, S, _ = x.shape
    h, kv, dh = spec.heads, spec.kv_heads, spec.d // spec.heads
    out = np.zeros((B, S, spec.d))
    bucket = L.distance_buckets(S, spec.buckets, spec.max_distance) if spec.buckets else None
    for b in range(B):
        for a in range(h):
            g = a // (h // kv)
            q, k, v = (x[b, :, at * dh:(at + 1) * dh] for at in (a, h + g, h + kv + g))
            for i in range(S):
                seen = [j for j in range(i + 1) if not spec.window or i - j < spec.window or j < spec.sinks]
                s = np.array([q[i] @ k[j] / math.sqrt(dh) + (table[a, bucket[i - j]] if spec.buckets else 0.0) for j in seen])
                e = np.exp(s - s.max())
                out[b, i, a * dh:(a + 1) * dh] = (e / e.sum()) @ v[seen]
    return out


SPECS = [W.LocalAttention(12, 2, 9, 2), W.LocalAttention(12, 4, 9, 2, window=3), W.LocalAttention(12, 4, 11, 1, window=2, sinks=3),
         W.LocalAttention(6, 2, 1, 1, window=1, sinks=1, buckets=4, max_distance=9), W.LocalAttention(12, 4, 13, 4, 0, 0, 5, 8),
         W.LocalAttention(12, 6, 14, 3, window=5, sinks=1, buckets=6, max_distance=7)]


@pytest.mark.parametrize("spec", SPECS, ids=str)
def test_windowed_attention_forward_brute_force(spec):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2,) + spec.in_shape())
    table = rng.standard_normal((spec.heads, spec.buckets))
    assert np.allclose(L.local_attention_forward(x, spec, table), _loops(x, spec, table), atol=1e-12)


def test_without_window_and_bias_it_is_causal_attention():
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 7, 36)), rng.standard_normal((2, 7, 12))
    spec = W.LocalAttention(12, 3, 7, 3)
    assert np.allclose(L.local_attention_forward(x, spec), L.attention_forward(x, 3), atol=1e-13)
    dx, dtable = L.local_attention_backward(dy, x, spec)
    assert dtable is None and np.allclose(dx, L.attention_backward(dy, x, 3), atol=1e-13)


@pytest.mark.parametrize("spec", SPECS, ids=str)
def test_windowed_attention_backward_finite_differences(spec):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((2,) + spec.in_shape())
    table = rng.standard_normal((spec.heads, spec.buckets))
    c = rng.standard_normal((2,) + spec.out_shape())
    f = lambda x, t: float((L.local_attention_forward(x, spec, t) * c).sum())
    dx, dtable = L.local_attention_backward(c, x, spec, table)
    eps = 1e-6
    for grad, at in [(dx, x)] + ([(dtable, table)] if spec.buckets else []):
        for _ in range(25):
            i = tuple(rng.integers(0, n) for n in at.shape)
            keep = at[i]
            at[i] = keep + eps
            up = f(x, table)
            at[i] = keep - eps
            down = f(x, table)
            at[i] = keep
            assert abs((up - down) / (2 * eps) - grad[i]) <= 1e-7 * (1 + abs(grad[i]))


def test_the_backward_pass_keeps_the_table_of_its_forward_pass():
    """Under every policy: the probabilities are the forward pass's, whatever the table has become since."""
    spec = W.LocalAttention(8, 2, 6, 2, 4, 1, 4, 6)
    rng = np.random.default_rng(4)
    x, dy, table = rng.standard_normal((2, 6, 24)), rng.standard_normal((2, 6, 8)), rng.standard_normal((2, 4))
    for policy in ("latest", "convex", "eq1", "stashed"):
        st = Stage((spec,), [table, np.zeros(0)], policy=policy, lam=0.3, lr=0.5, momentum=0.0, n=1)
        st.forward(0, 0, x)
        st.forward(1, 0, x)
        st.backward(0, dy)
        st.update(0)
        dx = st.backward(1, dy)
        want, dtable = L.local_attention_backward(dy, x, spec, table)
        assert np.allclose(dx.reshape(want.shape), want) and np.allclose(st.g[0], dtable)


def test_distillation_closed_forms_and_finite_differences():
    rng = np.random.default_rng(5)
    z = rng.standard_normal((4, 9))
    labels = np.array([3, 0, 8, 3])
    # labels alone: cross-entropy
    loss, dz = L.distill_loss(z, np.zeros((4, 1)), np.full((4, 1), -1), 2.0, labels, 1.0)
    want, dwant = L.softmax_cross_entropy(z, labels, 4)
    assert abs(loss - want) < 1e-13 and np.allclose(dz, dwant, atol=1e-14)
    # a teacher that says what the student says: no loss, no gradient
    ids = np.tile(np.arange(9), (4, 1))
    loss, dz = L.distill_loss(z, z.copy(), ids, 3.0, labels, 0.0)
    assert abs(loss) < 1e-14 and np.abs(dz).max() < 1e-15
    # an entry twice, absent ones, a row without any, entries of -inf
    ids = np.array([[1, 4, 4], [2, -1, -1], [-1, -1, -1], [0, 5, 7]])
    teacher = rng.standard_normal((4, 3))
    teacher[3, 1] = -np.inf
    for temperature, weight in ((1.0, 0.0), (2.5, 0.3)):
        f = lambda z: L.distill_loss(z, teacher, ids, temperature, labels, weight)
        _, dz = f(z)
        for r in range(4):
            for c in range(9):
                up, down = z.copy(), z.copy()
                up[r, c] += 1e-6
                down[r, c] -= 1e-6
                assert abs((f(up)[0] - f(down)[0]) / 2e-6 - dz[r, c]) < 1e-8
        assert np.abs(dz[2]).max() > 0 if weight else np.abs(dz[2]).max() == 0
