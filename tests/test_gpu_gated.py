"""The gated layer, act(z_2f) z_2f+1 with z = x W^T + b, forward and backward, against fp64.

Every result is held to a bound of its own, formed in fp64 from the operations that lead to it.  Units: f = 2^-24, u = f in fp32 and 2^-8 in
bf16 (what a stored value is off at most, relative).
  z      (K + 2) f (sum |x||W| + |b|): products of bf16 values are exact in fp32, sums are chains over K
  act    its slope (below 1.13) times that, and 16 f (1 + |z|) for its evaluation; the same for act', whose slope is below 0.8; a ReLU's
         derivative is either where |z| is within its error
  y, and what is kept for the backward pass   the factors' errors times the other factor, 2 f, and u for the stored value
  dz     |dy| times what was kept is off, and u;  dx, dW, db: that summed, and one f for every term of a sum"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
F = 2.0 ** -24
U = {"f32": F, "bf16": 2.0 ** -8}


def _stage(layers, params, dtype, mb, n=1, needs_dx=True, lr=0.0, policy="latest", **more):
    from paper_2509_23241_amd.runner import GpuStage
    return GpuStage(layers, params, dtype=dtype, mb=mb, n=n, stage_index=1, num_stages=2, policy=policy, lam=0.1, lr=lr, momentum=0.0,
                    needs_dx=needs_dx, **more)


def _inputs(seqs, tokens, d, f, dtype, seed=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + seqs + 7 * tokens + d + 3 * f)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")
    return (normal(seqs, tokens * d).to(t), normal(seqs, tokens * f).to(t), (normal(2 * f, d) * 1.5 / d ** 0.5).to(t).float(),
            0.3 * normal(2 * f))


def _act(z, act):
    import torch
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(z / 2 ** 0.5))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / (2 * np.pi) ** 0.5
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    return z, torch.ones_like(z)


def _reference(x, dy, w, b, act, dtype):
    """{name: (value, bound)} in fp64."""
    import torch
    u, (n2, d) = U[dtype], w.shape
    x, dy, w, b = x.double().view(-1, d), dy.double().view(-1, n2 // 2), w.double(), b.double()
    rows = x.shape[0]
    z = x @ w.t() + b
    ez = (d + 2) * F * (x.abs() @ w.abs().t() + b.abs())
    gate, up, eg, eu = z[:, 0::2], z[:, 1::2], ez[:, 0::2], ez[:, 1::2]
    a, slope = _act(gate, act)
    evaluated = 16 * F * (1 + gate.abs()) if act in ("silu", "gelu") else 0.0
    ea = 1.13 * eg + evaluated
    es = 0.8 * eg + evaluated if act in ("silu", "gelu") else (gate.abs() <= eg).double() if act == "relu" else torch.zeros_like(eg)
    y, c = a * up, up * slope
    ey = up.abs() * ea + (a.abs() + ea) * eu + (2 * F + u) * y.abs()
    ec = up.abs() * es + (slope.abs() + es) * eu + (2 * F + u) * c.abs()
    kept = lambda p, q: torch.stack([p, q], 2).view(rows, n2)
    dz = kept(dy * c, dy * a)
    edz = kept(dy.abs() * ec, dy.abs() * (ea + u * a.abs())) + (u + F) * dz.abs()
    edz = edz * (1 + u)
    dx, dw, db = dz @ w, dz.t() @ x, dz.sum(0)
    out = {"y": (y, ey * (1 + u)), "dx": (dx, edz @ w.abs() + (n2 + 2) * F * (dz.abs() @ w.abs()) + u * dx.abs()),
           "dw": (dw, edz.t() @ x.abs() + (rows + 8) * F * (dz.abs().t() @ x.abs())),
           "db": (db, edz.sum(0) + (rows + 8) * F * dz.abs().sum(0))}
    return out


def _run(x, dy, w, b, act, dtype, tokens, n=1, minibatch=False, shift=0):
    """One stage of this layer; shift: values by which the caller's tensors are off a 16-byte address."""
    import torch
    d, f = w.shape[1], w.shape[0] // 2
    seqs = x.shape[0]
    st = _stage([("gated", d, f, act, tokens)], [w.cpu().numpy(), b.cpu().numpy()], dtype, seqs // n, n)

    def off(t):
        flat = torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")
        out = flat[shift: shift + t.numel()].view(t.shape)
        out.copy_(t)
        return out
    x, dy, y, dx = off(x), off(dy), off(torch.empty_like(dy)), off(torch.empty_like(x))
    if minibatch:
        st.forward_minibatch(0, x, y)
    else:
        k = seqs // n
        for ub in range(n):
            st.forward(0, ub, x[ub * k:(ub + 1) * k], y[ub * k:(ub + 1) * k])
    st.backward(0, dy, dx)
    wo, bo = st.sizes.w_offset[0], st.sizes.b_offset[0]
    out = {"y": y.clone().view(-1, f), "dx": dx.clone().view(-1, d), "dw": st.grad[wo: wo + w.numel()].clone().view_as(w),
           "db": st.grad[bo: bo + b.numel()].clone()}
    st.close()
    return out


def _check(got, want, name=""):
    import torch
    for k, (ref, bound) in want.items():
        a = got[k].double()
        assert bool(torch.isfinite(a).all()), (name, k)
        over = float(((a - ref).abs() / (bound + 1e-30)).max())
        print(name, k, "share of its bound %.3g" % over, "rel %.2e" % float((a - ref).norm() / ref.norm().clamp(min=1e-300)))
        assert over <= 1.0, (name, k, over)


SIZES = [(1, 1, 1, 1), (1, 1, 8, 4), (1, 1, 512, 1408), (3, 1, 7, 5), (2, 9, 16, 3), (1, 33, 24, 12), (5, 13, 40, 17), (2, 50, 64, 64),
         (1, 64, 72, 100), (1, 127, 130, 66), (1, 129, 128, 128), (4, 100, 96, 250), (3, 85, 100, 36), (1, 700, 256, 340), (2, 300, 200, 641),
         (1, 1024, 512, 512), (4, 333, 512, 1365), (1, 2048, 264, 1000), (1, 4096, 64, 130), (1, 5000, 320, 68)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,tokens,d,f", SIZES)
def test_against_fp64(seqs, tokens, d, f, dtype):
    x, dy, w, b = _inputs(seqs, tokens, d, f, dtype)
    for act in ("silu", "gelu", "relu", "none") if seqs * tokens < 1000 else ("silu",):
        _check(_run(x, dy, w, b, act, dtype, tokens), _reference(x, dy, w, b, act, dtype), act)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,tokens,d,f", [(2, 9, 16, 3), (2, 50, 64, 64), (3, 85, 100, 36), (1, 300, 512, 640)])
def test_tensors_at_odd_addresses(seqs, tokens, d, f, dtype):
    x, dy, w, b = _inputs(seqs, tokens, d, f, dtype)
    for shift in (1, 2, 4):
        _check(_run(x, dy, w, b, "silu", dtype, tokens, shift=shift), _reference(x, dy, w, b, "silu", dtype), shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,tokens,d,f", [(6, 5, 32, 20), (6, 50, 64, 96), (6, 3, 24, 7)])
def test_micro_batches_give_the_same_bits(seqs, tokens, d, f, dtype):
    import torch
    x, dy, w, b = _inputs(seqs, tokens, d, f, dtype)
    whole = _run(x, dy, w, b, "silu", dtype, tokens)
    for n, minibatch in ((1, False), (2, False), (3, True), (6, False)):
        again = _run(x, dy, w, b, "silu", dtype, tokens, n=n, minibatch=minibatch)
        for k in whole:
            assert torch.equal(whole[k], again[k]), (n, minibatch, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_gates(dtype):
    """Gates of thousands either way: activations and slopes at their limits, nothing overflows on the way."""
    import torch
    x, dy, w, b = _inputs(1, 40, 16, 24, dtype)
    x = x.sign() * 512
    for act in ("silu", "gelu", "relu"):
        _check(_run(x, dy, w, b, act, dtype, 40), _reference(x, dy, w, b, act, dtype), act)


def test_gradient_against_differences():
    """What sum(y dy) changes by over a step of the weights either way, against the gradient times the step.  Allowed: what the outputs and
    the gradient are off by their bounds, and what the step's own curvature is in fp64.  (In bf16 the outputs' rounding alone, summed up,
    is more than the change: 2^-8 sum |y dy| for 600 outputs of order one.)"""
    import torch
    dtype = "f32"
    x, dy, w, b = _inputs(1, 30, 24, 20, dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    direction = torch.randn(w.shape, generator=g, device="cuda") / w.numel() ** 0.5
    sides = [(w + s * direction).to(x.dtype).float() for s in (0.25, -0.25)]
    step = (sides[0] - sides[1]).double()
    d2 = dy.double().view(30, 20)
    change, exact, allowed = 0.0, 0.0, 0.0
    for w2, sign in zip(sides, (1, -1)):
        y, ey = _reference(x, dy, w2, b, "silu", dtype)["y"]
        change += sign * float((_run(x, dy, w2, b, "silu", dtype, 30)["y"].double() * d2).sum())
        exact += sign * float((y * d2).sum())
        allowed += float((ey * d2.abs()).sum())
    dw, edw = _reference(x, dy, w, b, "silu", dtype)["dw"]
    got = float((_run(x, dy, w, b, "silu", dtype, 30)["dw"].double() * step).sum())
    allowed += float((edw * step.abs()).sum()) + abs(exact - float((dw * step).sum()))
    assert abs(change - got) <= allowed, (change, got, allowed)
    assert allowed < 0.5 * abs(got)                      # and the step is one that a wrong gradient would not pass


def test_update_and_versions_follow_the_oracle():
    """Decoder blocks with gated halves, with staleness, under every policy; gated layers one behind another, first and last in a stage."""
    from stage_parity import run_stage
    from synth_inputs import workloads as W
    t, d = 10, 32
    block = (W.Residual(d, t, "begin"), W.LayerNorm(d, t), W.Gated(d, 40, "silu", t), W.Dense(40, d, "none", tokens=t), W.Residual(d, t, "add"))
    row = (W.Gated(d, 24, "gelu", t), W.Gated(24, 36, "none", t), W.Dense(36, 16, "gelu", tokens=t), W.Gated(16, 6, "silu", t))
    for dtype in ("f32", "bf16"):
        for policy in ("convex", "latest", "stashed", "eq1"):
            print(dtype, policy, run_stage(block, f"gated_{dtype}", dtype, mb=2, n=2, policy=policy))
    # Three products of gates in a row and no normalisation: at the driver's step of 0.05 the exact weights leave fp32's range.  In bf16
    # every product adds up what its factors were rounded by (the oracle's two precisions are 3 % apart by the fourth mini-batch): the
    # next test compares bits there.
    print(run_stage(row, "gated_row_f32", "f32", mb=2, n=2, lr=0.002, mean_loss_dy=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_layers_in_a_row_are_those_of_single_stages(dtype):
    import torch
    t = 10   # (the dense layer has no activation: within a stage the gradient passes one before it is rounded, between stages behind)
    layers = [("gated", 32, 24, "gelu", t), ("gated", 24, 36, "none", t), (36, 16, "none", t), ("gated", 16, 6, "silu", t)]
    rng = np.random.default_rng(2)
    params = [[rng.standard_normal((2 * l[2], l[1])).astype(np.float32) * 0.4, rng.standard_normal(2 * l[2]).astype(np.float32) * 0.1]
              if l[0] == "gated" else [rng.standard_normal((16, 36)).astype(np.float32) * 0.2, rng.standard_normal(16).astype(np.float32) * 0.1]
              for l in layers]
    x, _, _, _ = _inputs(4, t, 32, 6, dtype)
    _, dy, _, _ = _inputs(4, t, 16, 6, dtype)

    def run(stages):
        sts = [_stage(ls, ps, dtype, 4) for ls, ps in stages]
        a = x
        for st in sts:
            a = st.forward(0, 0, a)[0]
        out, g = [a.clone()], dy
        for st in reversed(sts):
            g = st.backward(0, g)[0]
        out += [g.clone(), torch.cat([st.grad[: st.P] for st in sts])]
        for st in sts:
            st.close()
        return out
    for a, b in zip(run([(layers, sum(params, []))]), run([([l], p) for l, p in zip(layers, params)])):
        if a.dtype == torch.float32 and a.dim() == 1:      # sums over rows may be cut up otherwise behind a layer of the same stage
            assert float((a - b).abs().max()) <= 64 * F * float(a.abs().max())
        else:
            assert torch.equal(a, b)


@pytest.mark.parametrize("needs_dx", [True, False])
def test_first_layer_without_an_input_gradient(needs_dx):
    import torch
    x, dy, w, b = _inputs(2, 20, 32, 24, "bf16")
    st = _stage([("gated", 32, 24, "silu", 20)], [w.cpu().numpy(), b.cpu().numpy()], "bf16", 2, needs_dx=needs_dx)
    st.forward(0, 0, x)
    dx, _ = st.backward(0, dy)
    assert (dx is None) == (not needs_dx)
    want = _reference(x, dy, w, b, "silu", "bf16")
    wo = st.sizes.w_offset[0]
    _check({"dw": st.grad[wo: wo + w.numel()].view_as(w)}, {"dw": want["dw"]})
    st.close()
