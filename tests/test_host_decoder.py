"""Descriptions of gated and rotary layers and calls of the losses on log probabilities that the library takes or refuses; no GPU needed."""
import ctypes as C

import pytest

from paper_2509_23241_amd import binding as B

GOOD = dict(dtype="bf16", mb=2, n=3, stage_index=1, num_stages=4, ring_capacity=3, max_in_flight=3, policy="convex", needs_dx=True,
            lam=0.1, lr=0.01, momentum=0.9)
NAN, INF = float("nan"), float("inf")


def _query(layers, **changed):
    return B.stage_workspace_query(B.make_desc(layers, **{**GOOD, **changed}))


def test_descriptions_that_are_taken():
    for dtype in ("f32", "bf16"):
        s = _query([("gated", 16, 24, "silu", 5)], dtype=dtype)
        assert s.w_offset[0] == 0 and s.b_offset[0] == 48 * 16 and s.param_count == 48 * 16 + 64
        for act in ("none", "relu", "gelu", "silu"):
            _query([("gated", 7, 3, act, 1)], dtype=dtype)
        assert _query([("rotary", 4, 2, 16, 8, 16, "halves")], dtype=dtype).param_count == 0
    for heads, kv, dh, rotated in ((1, 1, 2, 2), (16, 4, 128, 128), (3, 3, 5, 4), (1, 1, 256, 256), (7, 1, 96, 2)):
        for layout in ("pairs", "halves"):
            _query([("rotary", heads, kv, dh, 9, rotated, layout)])
    for more in ((1.0,), (500000.0, 2 ** 31 - 9), (10000.0, 0, 0.25), (10000.0, 0, 8.0, 8192, 0.0, 1.0), (10000.0, 0, 8.0, 8192, 1.0, 4.0, 0.5)):
        _query([("rotary", 4, 2, 16, 8, 16, "halves") + more])


def test_the_description_keeps_its_size():
    assert C.sizeof(B.tp_layer_desc) == 4 * (4 + 5 + 7)


def test_what_a_turn_in_place_saves():
    front, att, back = (8, 64, "none", 6), ("local", 32, 2, 6, 1, 3, 1), (32, 8, "none", 6)
    turn = ("rotary", 2, 1, 16, 6, 16, "halves")
    plain = _query([front, att, back]).act_bytes
    assert _query([front, turn, att, back]).act_bytes == plain
    kept = 3 * 6 * 2 * 3 * 64 * 2                          # in flight, samples, tokens, values
    for layers in ([("ln", 64, 6), turn, att, back], [(8, 64, "gelu", 6), turn, att, back], [front, turn, (64, 8, "none", 6)]):
        without = [l for l in layers if l is not turn]
        assert _query(layers).act_bytes - _query(without).act_bytes >= 3 * 6 * 6 * 64 * 2, layers
    assert kept > 0


@pytest.mark.parametrize("layer", [
    ("gated", 16, 24, "silu", 0), ("gated", 0, 24, "silu", 5), ("gated", 16, 0, "silu", 5), ("gated", 16, 24, 4, 5), ("gated", 16, 24, -1, 5),
    ("gated", 8, 1 << 28, "silu", 4),                   # a sample too large
    ("rotary", 4, 2, 16, 0, 16, "halves"), ("rotary", 0, 2, 16, 8, 16, "halves"), ("rotary", 4, 0, 16, 8, 16, "halves"),
    ("rotary", 4, 2, 16, 8, 0, "halves"), ("rotary", 4, 2, 16, 8, 15, "halves"), ("rotary", 4, 2, 16, 8, 18, "halves"),
    ("rotary", 4, 2, 16, 8, -2, "halves"), ("rotary", 4, 2, 257, 8, 256, "halves"), ("rotary", 4, 2, 16, 8, 16, 2), ("rotary", 4, 2, 16, 8, 16, -1),
    ("rotary", 4, 2, 16, 8, 16, "halves", 0.0), ("rotary", 4, 2, 16, 8, 16, "halves", NAN), ("rotary", 4, 2, 16, 8, 16, "halves", INF),
    ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, -1), ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 2 ** 31 - 8),
    ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, 0.0), ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, -2.0),
    ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, 8.0, -1, 1.0, 4.0), ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, 8.0, 64, 4.0, 4.0),
    ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, 8.0, 64, -1.0, 4.0), ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, 8.0, 64, 1.0, INF),
    ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, 8.0, 0, 1.0, 4.0),      # by parts without an original length
    ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, 1.0, 0, 0.0, 0.0, 0.0), ("rotary", 4, 2, 16, 8, 16, "halves", 1e4, 0, 1.0, 0, 0.0, 0.0, NAN),
], ids=str)
def test_descriptions_that_are_refused(layer):
    with pytest.raises(B.StageLibError) as e:
        _query([layer])
    assert e.value.code == B.TP_EINVAL


def test_malformed_fields_are_refused():
    gated, turn = ("gated", 16, 24, "silu", 5), ("rotary", 4, 2, 16, 8, 16, "halves")
    for layer, changes in ((gated, (lambda L: L.geom.__setitem__(1, 1), lambda L: L.rel.__setitem__(0, 1), lambda L: L.reserved.__setitem__(0, 1),
                                    lambda L: L.rope.__setitem__(4, 1.0))),
                           (turn, (lambda L: setattr(L, "act", B.TP_ACT_RELU), lambda L: setattr(L, "in_features", 127),
                                   lambda L: setattr(L, "out_features", 64), lambda L: L.geom.__setitem__(2, 2 ** 31 - 1)))):
        B.stage_workspace_query(B.make_desc([layer], **GOOD))
        for change in changes:
            d = B.make_desc([layer], **GOOD)
            change(d.layers[0])
            with pytest.raises(B.StageLibError) as e:
                B.stage_workspace_query(d)
            assert e.value.code == B.TP_EINVAL
    for act in (B.TP_ACT_SILU, 4):                       # SiLU is the gated layer's
        with pytest.raises(B.StageLibError):
            _query([(8, 8, act)])
    with pytest.raises(B.StageLibError):                 # the layers' sizes have to chain
        _query([gated, (48, 8, "none", 5)])
    for layer in (gated, turn):                          # the rows of a mini-batch stay countable
        with pytest.raises(B.StageLibError):
            _query([layer[:4] + (1 << 20,) + layer[5:] if layer is turn else layer[:4] + (1 << 20,)], mb=1 << 12, n=1)


def _dry(layers, **changed):
    st = B.stage_init(B.make_desc(layers, **{**GOOD, "n": 1, "max_in_flight": 1, "ring_capacity": 1, "policy": "latest", **changed}), None, 0)
    return st


def test_loss_refusals():
    """On stages without device buffers, which check and launch nothing."""
    policy = lambda st, mb=0, low=0.2, high=0.2, kl=0.0: B.stage_loss_policy(st, mb, 0, 0, 0, 0, 0, 0, low, high, kl, 0, 0, 0)
    pairs = lambda st, mb=0, beta=0.1, smooth=0.0: B.stage_loss_preference(st, mb, 0, 0, 0, 0, beta, smooth, 0, 0, 0)
    st = _dry([(8, 10, "none", 3)])
    for call in (policy, pairs):
        with pytest.raises(B.StageLibError) as e:
            call(st)
        assert e.value.code == B.TP_ESTATE               # nothing forwarded yet
    B.stage_logprobs(st, 0, 0, 5, 0)                     # of any pass
    B.stage_forward(st, 0, 0, 0, 0)
    for good in (dict(), dict(low=0.0, high=0.0), dict(low=1.0, high=1e6, kl=1e6)):
        policy(st, **good)
    for good in (dict(), dict(beta=0.0, smooth=1.0), dict(beta=1e6)):
        pairs(st, **good)
    for bad in (dict(low=-0.1), dict(low=1.1), dict(low=NAN), dict(high=-0.1), dict(high=2e6), dict(high=NAN), dict(kl=-1.0), dict(kl=2e6), dict(kl=NAN)):
        with pytest.raises(B.StageLibError) as e:
            policy(st, **bad)
        assert e.value.code == B.TP_EINVAL, bad
    for bad in (dict(beta=-0.1), dict(beta=2e6), dict(beta=NAN), dict(smooth=-0.1), dict(smooth=1.1), dict(smooth=NAN)):
        with pytest.raises(B.StageLibError) as e:
            pairs(st, **bad)
        assert e.value.code == B.TP_EINVAL, bad
    for call in (policy, pairs):
        with pytest.raises(B.StageLibError) as e:
            call(st, mb=7)
        assert e.value.code == B.TP_ESTATE
    with pytest.raises(B.StageLibError) as e:
        B.stage_logprobs(st, 0, 0, 1 << 31, 0)
    assert e.value.code == B.TP_EINVAL
    B.stage_destroy(st)
    st = _dry([(8, 10, "none")], mb=3)                   # an odd number of samples makes no pairs
    B.stage_forward(st, 0, 0, 0, 0)
    policy(st)
    with pytest.raises(B.StageLibError) as e:
        pairs(st)
    assert e.value.code == B.TP_EINVAL
    B.stage_destroy(st)
    st = _dry([("gated", 8, 8, "silu", 1)])              # the losses need a dense last layer
    B.stage_forward(st, 0, 0, 0, 0)
    for call in (policy, pairs, lambda s: B.stage_logprobs(s, 0, 0, 1, 0)):
        with pytest.raises(B.StageLibError) as e:
            call(st)
        assert e.value.code == B.TP_EINVAL
    B.stage_destroy(st)


def test_rows_of_a_gated_layer():
    _query([("gated", 1, 1, "silu", 1 << 20)], mb=256, n=1)
    with pytest.raises(B.StageLibError) as e:
        _query([("gated", 1, 1, "silu", (1 << 20) + 1)], mb=256, n=1)
    assert e.value.code == B.TP_EINVAL
