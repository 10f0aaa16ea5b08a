"""Rotary positions, forward and backward, against fp64.

Bound: an angle is off by 2^-51 of itself (the speed's and the product's rounding in fp64) and 2^-25 by its reduced form in fp32; sine and
cosine of it by two ulps, their product with the amplitude by one: each is off amplitude * (4 f + 2^-25 + 2^-51 angle) + f.  The
turned value adds f for either product and the sum, and u for the stored value (f = 2^-24, u = f in fp32, 2^-8 in bf16).  What is not turned
keeps its bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
F = 2.0 ** -24
U = {"f32": F, "bf16": 2.0 ** -8}


def _spec(tokens, heads=2, kv=1, head=16, rotated=16, layout="halves", **more):
    from synth_inputs import workloads as W
    return W.Rotary(heads, kv, head, tokens, rotated, layout, **more)


def _stage(specs, dtype, mb, n=1, **more):
    from paper_2509_23241_amd.runner import GpuStage, layer_tuple
    return GpuStage([layer_tuple(s) for s in specs], [], dtype=dtype, mb=mb, n=n, stage_index=1, num_stages=2, policy="latest", lam=0.1,
                    lr=0.0, momentum=0.0, **more)


def _inputs(spec, seqs, dtype, seed=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + spec.tokens + seqs)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    return [torch.randn(seqs, spec.out_dim(), generator=g, device="cuda").to(t) for _ in range(2)]


def _reference(spec, x, back, dtype):
    """(value, bound, what is turned) in fp64."""
    import torch
    from oracle.layers import rotary_speeds
    seqs = x.shape[0]
    v = x.double().view(seqs, spec.tokens, -1, spec.head)
    half, heads = spec.rotated // 2, spec.heads + spec.kv_heads
    speeds = torch.from_numpy(rotary_speeds(spec)).cuda()
    angle = ((torch.arange(spec.tokens, device="cuda") + spec.first).double()[:, None] * speeds)[None, :, None]
    one = slice(0, half) if spec.layout == "halves" else slice(0, spec.rotated, 2)
    two = slice(half, spec.rotated) if spec.layout == "halves" else slice(1, spec.rotated, 2)
    a, b = v[:, :, :heads, one], v[:, :, :heads, two]
    amp = float(np.float32(spec.amplitude))
    c, s = amp * angle.cos(), amp * angle.sin() * (-1 if back else 1)
    off = amp * (4 * F + 2.0 ** -25 + 2.0 ** -51 * angle.abs()) + F * amp
    want, bound, turned = v.clone(), torch.zeros_like(v), torch.zeros(v.shape, dtype=torch.bool, device="cuda")
    for at, p, q in ((one, a * c, -b * s), (two, a * s, b * c)):
        want[:, :, :heads, at] = p + q
        bound[:, :, :heads, at] = (a.abs() + b.abs()) * off + 2 * F * (p.abs() + q.abs()) + U[dtype] * (p + q).abs()
        turned[:, :, :heads, at] = True
    return want.view(seqs, -1), (bound * (1 + U[dtype])).view(seqs, -1), turned.view(seqs, -1)


def _compare(spec, x, got, back, dtype, name=""):
    import torch
    want, bound, turned = _reference(spec, x, back, dtype)
    over = float(((got.double() - want).abs() / (bound + 1e-30))[turned].max())
    print(name, "backward" if back else "forward", "share of its bound %.3g" % over)
    assert over <= 1.0, (name, back, over)
    assert torch.equal(got[~turned], x[~turned])


SPECS = [
    _spec(1, head=2, rotated=2), _spec(1, heads=16, kv=4, head=128, rotated=128, first=100000, factor=8.0, original=8192, low=1.0, high=4.0, amplitude=1.125),
    _spec(2, heads=3, kv=3, head=5, rotated=4, layout="pairs"), _spec(7, head=20, rotated=6), _spec(7, head=20, rotated=20, layout="pairs"),
    _spec(33, heads=4, kv=2, head=64, rotated=64), _spec(33, heads=4, kv=2, head=64, rotated=32, layout="pairs", factor=4.0),
    _spec(50, heads=6, kv=2, head=80, rotated=40), _spec(50, heads=6, kv=2, head=80, rotated=80, layout="pairs", base=500000.0),
    _spec(129, heads=7, kv=1, head=96, rotated=48, amplitude=0.75), _spec(65, heads=2, kv=2, head=256, rotated=256, first=12345),
    _spec(65, heads=1, kv=1, head=256, rotated=130, layout="pairs"), _spec(300, heads=8, kv=8, head=32, rotated=16, original=64, factor=2.0, low=0.5, high=3.0),
    _spec(1000, heads=16, kv=16, head=128, rotated=128), _spec(1025, heads=4, kv=1, head=72, rotated=24, layout="pairs"),
    _spec(700, heads=32, kv=8, head=64, rotated=64, layout="pairs"), _spec(4100, heads=2, kv=1, head=64, rotated=64, first=1 << 24),
    _spec(9, heads=2, kv=1, head=16, rotated=16, first=2 ** 31 - 10), _spec(70, head=24, rotated=24, base=1.0, factor=0.5),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spec", SPECS, ids=lambda s: "-".join(str(v) for v in list(s.__dict__.values())[:-2]))
def test_against_fp64(spec, dtype):
    for seqs in (1, 3) if spec.tokens < 1000 else (2,):
        x, dy = _inputs(spec, seqs, dtype)
        st = _stage([spec], dtype, seqs)
        y, _ = st.forward(0, 0, x)
        dx, _ = st.backward(0, dy)
        st.blend_update(0)
        _compare(spec, x, y, False, dtype, seqs)
        _compare(spec, dy, dx, True, dtype, seqs)
        st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spec", SPECS[3:9], ids=lambda s: "-".join(str(v) for v in list(s.__dict__.values())[:-2]))
def test_tensors_at_odd_addresses(spec, dtype):
    import torch
    x, dy = _inputs(spec, 2, dtype)
    st = _stage([spec], dtype, 2)
    for j, shift in enumerate((1, 2, 4)):
        place = lambda t: torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")[shift: shift + t.numel()].view(t.shape).copy_(t)
        y, dx = place(x), place(x)
        st.forward(j, 0, place(x), y)
        st.backward(j, place(dy), dx)
        st.blend_update(j)
        _compare(spec, x, y, False, dtype, shift)
        _compare(spec, dy, dx, True, dtype, shift)
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_turn_keeps_lengths_and_distances(dtype):
    """What the layer is for: scores of turned queries and keys depend on their distance alone.  Each turned value of a head of 64 is off
    its bound, so a score is off by at most those times the other side's values."""
    import torch
    for layout in ("halves", "pairs"):
        spec = _spec(400, heads=1, kv=1, head=64, rotated=64, layout=layout)
        x, _ = _inputs(spec, 1, dtype)
        x = x.view(400, 3, 64)[:1].expand(400, 3, 64).contiguous().view(1, -1)      # one query and key at every position
        st = _stage([spec], dtype, 1)
        y, _ = st.forward(0, 0, x)
        _, bound, _ = _reference(spec, x, False, dtype)
        q, k = (y.double().view(400, 3, 64)[:, i] for i in (0, 1))
        eq, ek = (bound.view(400, 3, 64)[:, i] for i in (0, 1))
        scores, off = q @ k.t().contiguous(), eq @ k.abs().t().contiguous() + (q.abs() + eq) @ ek.t().contiguous()
        for distance in (0, 1, 17, 200):
            along, slack = scores.diagonal(-distance), off.diagonal(-distance)
            assert float((along - along[0]).abs().max()) <= 2 * float(slack.max()), (layout, distance)
        st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("attention", ["attn", "local"])
def test_in_place_between_a_dense_layer_and_attention(attention, dtype):
    """The same bits as with the turn in a stage of its own, forward and backward, with and without forward streams; the plan keeps no second
    tensor for it."""
    import torch
    from paper_2509_23241_amd.runner import GpuStage, layer_tuple
    from synth_inputs import workloads as W
    t, heads, dh = 48, 4, 32
    d = heads * dh
    turn = _spec(t, heads=heads, kv=heads, head=dh, rotated=dh)
    front = (d, 3 * d, "none", t)
    att = ("attn", d, heads, t) if attention == "attn" else ("local", d, heads, t, heads, 20, 2)
    back = (d, 24, "none", t)
    rng = np.random.default_rng(3)
    w = [rng.standard_normal(s).astype(np.float32) * 0.1 for s in ((3 * d, d), (3 * d,), (24, d), (24,))]
    kw = dict(dtype=dtype, mb=2, n=2, stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn(4, t * d, generator=g, device="cuda").to(tt)
    dy = torch.randn(4, t * 24, generator=g, device="cuda").to(tt)

    def run(stages, **more):
        sts = [GpuStage(ls, ps, **kw, **more) for ls, ps in stages]
        for ub in range(2):
            a = x[2 * ub: 2 * ub + 2].contiguous()
            for st in sts:
                a = st.forward(0, ub, a)[0]
                st.forward_join()
            out = a if ub == 0 else torch.cat([out, a])
        grad = dy
        for st in reversed(sts):
            grad, _ = st.backward(0, grad)
        got = [out.clone(), grad.clone()] + [st.grad.clone() for st in sts if st.P]
        sizes = sum(st.sizes.act_bytes for st in sts)
        for st in sts:
            st.close()
        return got, sizes

    one, kept = run([([front, layer_tuple(turn), att, back], w)])
    apart, _ = run([([front], w[:2]), ([layer_tuple(turn)], []), ([att, back], w[2:])])
    assert torch.equal(one[0], apart[0]) and torch.equal(one[1], apart[1])
    assert torch.equal(one[2], torch.cat(apart[2:]))
    without, bare = run([([front, att, back], w)])
    assert kept == bare and not torch.equal(without[0], one[0])
    if attention == "local":
        streams, _ = run([([front, layer_tuple(turn), att, back], w)], forward_stream=2)
        for a, b in zip(one, streams):
            assert torch.equal(a, b)


def test_layers_beside_it():
    """Where the turn cannot be made in place: behind an activation, a residual begin, attention; in front of other layers; first and last."""
    from stage_parity import run_stage
    from synth_inputs import workloads as W
    t = 12
    turn = lambda layout="halves", **more: _spec(t, heads=2, kv=1, head=16, rotated=8, layout=layout, **more)
    for dtype in ("f32", "bf16"):
        specs = (turn(), W.Residual(64, t, "begin"), turn("pairs", first=5), W.Dense(64, 64, "gelu", tokens=t), turn(), W.LocalAttention(32, 2, t, 1, 6, 1),
                 W.Dense(32, 64, "none", tokens=t), W.Residual(64, t, "add"), W.Gated(64, 64, "silu", t), turn("pairs"), W.LayerNorm(64, t), turn())
        print(dtype, run_stage(specs, f"rotary_beside_{dtype}", dtype, mb=2, n=2, policy="convex", check_saved=False))
        specs = (W.Dense(24, 64, "relu", tokens=t), turn(), W.Dense(64, 64, "none", tokens=t), turn(), W.LocalAttention(32, 2, t, 1), W.Dense(32, 8, "none", tokens=t))
        print(dtype, run_stage(specs, f"rotary_relu_{dtype}", dtype, mb=2, n=2, policy="convex", check_saved=False, fixed_masks=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_micro_batches_give_the_same_bits(dtype):
    import torch
    spec = _spec(37, heads=4, kv=2, head=64, rotated=64)
    x, _ = _inputs(spec, 6, dtype)
    st = _stage([spec], dtype, 6)
    whole = st.forward(0, 0, x)[0].clone()
    st.close()
    for n in (2, 3):
        st = _stage([spec], dtype, 6 // n, n)
        parts = torch.cat([st.forward(0, ub, x[ub * 6 // n:(ub + 1) * 6 // n])[0] for ub in range(n)])
        assert torch.equal(whole, parts)
        st.close()
        st = _stage([spec], dtype, 6 // n, n)
        assert torch.equal(whole, st.forward_minibatch(0, x, torch.empty_like(x))[0])
        st.close()
