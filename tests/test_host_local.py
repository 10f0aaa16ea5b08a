"""Descriptions of windowed attention layers and calls of the distillation loss that the library takes or refuses; no GPU needed."""
import ctypes as C

import pytest

from paper_2509_23241_amd import binding as B

GOOD = dict(dtype="bf16", mb=2, n=3, stage_index=1, num_stages=4, ring_capacity=3, max_in_flight=3, policy="convex", needs_dx=True,
            lam=0.1, lr=0.01, momentum=0.9)


def _query(layers, **changed):
    return B.stage_workspace_query(B.make_desc(layers, **{**GOOD, **changed}))


def test_descriptions_that_are_taken():
    for dtype in ("f32", "bf16"):
        s = _query([("local", 32, 4, 8, 2, 3, 1, 6, 9)], dtype=dtype)
        assert s.param_count == 64 and s.w_offset[0] == 0          # 4 x 6 biases, padded; no second tensor behind them
        assert _query([("local", 32, 4, 8, 2, 3, 1)], dtype=dtype).param_count == 0
        s = _query([(16, 64, "none", 8), ("local", 32, 4, 8, 2, 0, 0, 6, 9), (32, 8, "none", 8)], dtype=dtype)
        assert s.w_offset[1] == 64 * 16 + 64 and s.w_offset[2] == s.w_offset[1] + 64
    for heads, kv, dh in ((1, 1, 1), (4, 4, 256), (16, 1, 128), (7, 7, 3), (6, 2, 80)):
        for tokens, window, sinks in ((1, 1, 1), (1, 0, 0), (1000, 1, 0), (1000, 5000, 2000), (30000, 512, 4)):
            _query([("local", heads * dh, heads, tokens, kv, window, sinks)])
    for buckets, reach in ((2, 2), (2, 1 << 20), (128, 65), (128, 1 << 20), (5, 3)):
        _query([("local", 32, 4, 8, 2, 3, 1, buckets, reach)])


def test_the_description_keeps_its_size():
    assert C.sizeof(B.tp_layer_desc) == 4 * (4 + 5 + 7)


@pytest.mark.parametrize("layer", [
    ("local", 32, 5, 8, 1, 3, 1),                       # heads do not divide the width
    ("local", 32, 4, 8, 3, 3, 1),                       # key heads do not divide the heads
    ("local", 32, 4, 8, 0, 3, 1),                       # no key heads
    ("local", 32, 4, 8, 8, 3, 1),                       # more key heads than heads
    ("local", 32, 4, 0, 4, 3, 1),                       # no tokens
    ("local", 32, 4, 8, 4, -1, 0), ("local", 32, 4, 8, 4, 3, -1),
    ("local", 32, 4, 8, 4, 0, 1),                       # first keys that stay visible beside no window
    ("local", 32, 4, 8, 4, 3, 1, 1, 9), ("local", 32, 4, 8, 4, 3, 1, 129, 900), ("local", 32, 4, 8, 4, 3, 1, -2, 9),
    ("local", 32, 4, 8, 4, 3, 1, 6, 3), ("local", 32, 4, 8, 4, 3, 1, 6, 0), ("local", 32, 4, 8, 4, 3, 1, 6, (1 << 20) + 1),
    ("local", 32, 4, 8, 4, 3, 1, 0, 9),                 # a reach without buckets
    ("local", 257, 1, 8, 1, 3, 1),                      # heads too wide
], ids=str)
def test_descriptions_that_are_refused(layer):
    with pytest.raises(B.StageLibError) as e:
        _query([layer])
    assert e.value.code == B.TP_EINVAL


def test_malformed_fields_are_refused():
    d = B.make_desc([("local", 32, 4, 8, 2, 3, 1, 6, 9)], **GOOD)
    B.stage_workspace_query(d)
    for change in (lambda L: setattr(L, "in_features", 95), lambda L: setattr(L, "act", B.TP_ACT_RELU),
                   lambda L: L.reserved.__setitem__(0, 1), lambda L: L.reserved.__setitem__(4, 1)):
        d = B.make_desc([("local", 32, 4, 8, 2, 3, 1, 6, 9)], **GOOD)
        change(d.layers[0])
        with pytest.raises(B.StageLibError):
            B.stage_workspace_query(d)
    d = B.make_desc([(8, 8, "none")], **GOOD)
    d.layers[0].rel[0] = 4                               # only windowed attention has a position bias
    with pytest.raises(B.StageLibError):
        B.stage_workspace_query(d)
    with pytest.raises(B.StageLibError):                 # the layers' sizes have to chain
        _query([(16, 96, "none", 8), ("local", 32, 4, 8, 2, 3, 1)])
    with pytest.raises(B.StageLibError):                 # the whole work of a call stays countable
        _query([("local", 32, 4, 8, 2, 3, 1)], mb=1 << 24, n=1)


def test_distillation_refusals():
    """On a stage without device buffers, which checks and launches nothing."""
    d = B.make_desc([(8, 10, "none")], **{**GOOD, "n": 1, "max_in_flight": 1, "ring_capacity": 1, "policy": "latest"})
    st = B.stage_init(d, None, 0)
    call = lambda k=3, t=1.0, w=0.5, mb=0: B.stage_loss_distill(st, mb, 0, 0, 0, k, t, 0, w, 0, 0)
    with pytest.raises(B.StageLibError) as e:
        call()
    assert e.value.code == B.TP_ESTATE                   # nothing forwarded yet
    B.stage_forward(st, 0, 0, 0, 0)
    call()
    call(k=1, t=1e-6, w=0.0)
    call(k=B.TP_MAX_TEACHER_ENTRIES, t=1e6, w=1.0)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(k=0), dict(k=-1), dict(k=B.TP_MAX_TEACHER_ENTRIES + 1), dict(t=0.0), dict(t=-1.0), dict(t=nan), dict(t=inf),
                dict(t=9e-7), dict(t=2e6), dict(w=-0.1), dict(w=1.1), dict(w=nan)):
        with pytest.raises(B.StageLibError) as e:
            call(**bad)
        assert e.value.code == B.TP_EINVAL, bad
    with pytest.raises(B.StageLibError) as e:
        call(mb=7)
    assert e.value.code == B.TP_ESTATE
    B.stage_destroy(st)
    st = B.stage_init(B.make_desc([("ln", 8, 1)], **{**GOOD, "n": 1}), None, 0)
    B.stage_forward(st, 0, 0, 0, 0)
    with pytest.raises(B.StageLibError) as e:
        call()
    assert e.value.code == B.TP_EINVAL                   # the loss needs a dense last layer
    B.stage_destroy(st)
