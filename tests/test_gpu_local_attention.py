"""Windowed attention with first keys that stay visible, shared key heads and a learned position bias, against fp64.

Every result is held to a bound of its own, formed in fp64 from the operations that lead to it.  Unit: 2^-24 in fp32; a bf16 value that
enters a product or is stored is off by 2^-8 of itself at most, products of bf16 values are exact in fp32.
  exponent   the dh terms of q.k and their sum, the bias, the maximum: E = (dh + 8) 2^-24 max(sum |q||k| / sqrt(dh) + |bias| + 1) log2(e)
  p          relative 2 E + (keys + 8) 2^-24
  y          sum of p |v| times that, and in bf16 of 2^-8 for the rounded p; 2^-8 |y| for the stored value
  dP         (dh + 8) 2^-24 sum |dy||v|;   delta  sum over p of what p and dP are off
  dS         p times (what dP and delta are off + |dP - delta| times what p is off)
  dq         its delta comes from the stored y, in bf16 2^-8 sum |dy||y| off; |dS| |k| 2^-8 for the rounded dS
  dk, dv     like y with dS and p; dtable: the sum of what dS is off and (pairs of a chain) 2^-24 |dS|."""
import math

import numpy as np
import pytest

from paper_2509_23241_amd import binding as B

pytestmark = pytest.mark.gpu
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _stage(c, params, n=1, lr=0.0, device="cuda:0", stream=None, needs_dx=True, policy="latest", layers=None, **more):
    from paper_2509_23241_amd.runner import GpuStage
    layer = ("local", c["heads"] * c["dh"], c["heads"], c["tokens"], c["kv"], c["window"], c["sinks"], c["buckets"], c["reach"])
    return GpuStage(layers or [layer], params, dtype=c["dtype"], mb=c["seqs"] // n, n=n, stage_index=1, num_stages=2, policy=policy,
                    lam=0.1, lr=lr, momentum=0.0, needs_dx=needs_dx, device=device, stream=stream, **more)


def _case(tokens, heads=2, dh=64, kv=2, window=0, sinks=0, buckets=0, reach=0, seqs=2, dtype="bf16"):
    return dict(tokens=tokens, heads=heads, dh=dh, kv=kv, window=window, sinks=sinks, buckets=buckets, reach=reach, seqs=seqs, dtype=dtype)


def _inputs(c, seed=0, device="cuda:0"):
    import torch
    g = torch.Generator(device=device)
    g.manual_seed(seed + c["tokens"])
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    width = (c["heads"] + 2 * c["kv"]) * c["dh"]
    x = torch.randn(c["seqs"], c["tokens"], width, generator=g, device=device).to(t)
    dy = torch.randn(c["seqs"], c["tokens"], c["heads"] * c["dh"], generator=g, device=device).to(t)
    table = torch.randn(c["heads"], c["buckets"], generator=g, device=device) if c["buckets"] else None
    return x, dy, table


def _params(table):
    return [] if table is None else [table.cpu().numpy(), np.zeros(0, np.float32)]


def _visible(c, device):
    import torch
    i = torch.arange(c["tokens"], device=device)[:, None]
    j = torch.arange(c["tokens"], device=device)[None]
    seen = j <= i
    if c["window"]:
        seen &= (i - j < c["window"]) | (j < c["sinks"])
    return seen, (i - j).clamp(min=0)


def _reference(c, x, dy, table):
    """{name: (value, bound)} in fp64."""
    import torch
    from oracle.layers import distance_buckets
    h, kv, dh, S, n = c["heads"], c["kv"], c["dh"], c["tokens"], x.shape[0]
    u, f = U[c["dtype"]], 2.0 ** -24
    rounded = u if c["dtype"] == "bf16" else 0.0
    parts = x.double().view(n, S, h + 2 * kv, dh).transpose(1, 2)
    spread = torch.arange(kv, device=x.device).repeat_interleave(h // kv)
    q, k, v = parts[:, :h], parts[:, h + spread], parts[:, h + kv + spread]
    do = dy.double().view(n, S, h, dh).transpose(1, 2)
    seen, distance = _visible(c, x.device)
    T = lambda a: a.transpose(-1, -2)
    s = q @ T(k) / math.sqrt(dh)
    size = q.abs() @ T(k.abs()) / math.sqrt(dh)
    if table is not None:
        bucket = torch.from_numpy(distance_buckets(S, c["buckets"], c["reach"])).to(x.device)
        bias = table.double()[:, bucket][:, distance]
        s, size = s + bias, size + bias.abs()
    s = s.masked_fill(~seen, -math.inf)
    p = s.softmax(-1)
    ep = p * (2 * (dh + 8) * f * 1.4427 * (float(size.max()) + 1) + (S + 8) * f)
    y = p @ v
    ey = ep @ v.abs() + rounded * (p @ v.abs()) + u * y.abs()
    dp = do @ T(v)
    edp = (dh + 8) * f * (do.abs() @ T(v.abs()))
    delta = (p * dp).sum(-1, keepdim=True)
    edelta = (ep * dp.abs() + p * edp).sum(-1, keepdim=True) + (S + 8) * f * (p * dp.abs()).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    eds = ep * (dp - delta).abs() + p * (edp + edelta)
    first = u * (do.abs() * (y.abs() + (p @ v.abs()))).sum(-1, keepdim=True)    # of the delta that dq is formed with
    sc = 1 / math.sqrt(dh)
    dq = sc * ds @ k
    edq = sc * ((eds + p * first + (rounded + (S + 8) * f) * (ds.abs() + p * first)) @ k.abs()) + u * dq.abs()
    share = lambda a: a.reshape(n, kv, h // kv, S, dh).sum(2)
    chain = (S * (h // kv) + 8) * f
    dk = share(sc * T(ds) @ q)
    edk = share(sc * T(eds + (rounded + chain) * ds.abs()) @ q.abs()) + u * dk.abs()
    dv = share(T(p) @ do)
    edv = share(T(ep + (rounded + chain) * p) @ do.abs()) + u * dv.abs()
    flat = lambda a: a.transpose(1, 2).reshape(n, S, -1)
    out = {"y": (flat(y), flat(ey)), "dq": (flat(dq), flat(edq)), "dk": (flat(dk), flat(edk)), "dv": (flat(dv), flat(edv))}
    if table is not None:
        one = (bucket[:, None] == torch.arange(c["buckets"], device=x.device)).double()
        pick = one[distance]                                                   # [S, S, buckets]
        total = lambda a: torch.stack([(a.sum(0) * (pick[:, :, b] * seen)).sum((1, 2)) for b in range(c["buckets"])], 1)
        out["dtable"] = (total(ds), total(eds + (S + 64) * f * ds.abs()))
    return out


def _split(c, y, dx, grad):
    h, kv, dh = c["heads"], c["kv"], c["dh"]
    dx = dx.reshape(-1, c["tokens"], (h + 2 * kv) * dh)
    out = {"y": y.reshape(-1, c["tokens"], h * dh), "dq": dx[..., : h * dh], "dk": dx[..., h * dh: (h + kv) * dh], "dv": dx[..., (h + kv) * dh:]}
    if c["buckets"]:
        out["dtable"] = grad[: h * c["buckets"]].view(h, c["buckets"])
    return out


def _run(c, x, dy, table, n=1):
    """One stage of this layer alone, on mini-batches of n micro-batches."""
    st = _stage(c, _params(table), n=n)
    rows = c["seqs"] // n
    y = [st.forward(0, ub, x[ub * rows:(ub + 1) * rows].reshape(rows, -1).contiguous())[0] for ub in range(n)]
    import torch
    dx, _ = st.backward(0, dy.reshape(c["seqs"], -1))
    out = {k: t.clone() for k, t in _split(c, torch.cat(y), dx, st.grad).items()}
    st.close()
    return out


def _check(got, want, name=""):
    import torch
    for k, (ref, bound) in want.items():
        a = got[k].double()
        assert bool(torch.isfinite(a).all()), (name, k)
        # what is not finite in the reference's own bounds never happens here; 1e-30: zeros
        over = float(((a - ref).abs() / (bound + 1e-30)).max())
        rel = float((a - ref).norm() / ref.norm().clamp(min=1e-300))
        print(name, k, "share of its bound %.3g" % over, "rel %.2e" % rel)
        assert over <= 1.0, (name, k, over)


SHAPES = [
    _case(1, seqs=3), _case(1, window=1, sinks=1, buckets=4, reach=8), _case(2, window=1), _case(3, heads=4, kv=1, window=2, sinks=1),
    _case(16, heads=4, kv=4, window=8, sinks=2), _case(31, window=5), _case(33, window=32, sinks=1), _case(63, dh=128, window=64),
    _case(64, window=63, sinks=64), _case(65, dh=128, window=1, sinks=1), _case(96, window=33, sinks=31, buckets=32, reach=128),
    _case(127, heads=4, kv=2, dh=32, window=40, sinks=3), _case(128, dh=128, heads=4, kv=1, window=64, buckets=8, reach=20),
    _case(129, dh=80, heads=6, kv=2, window=100, sinks=70), _case(200, heads=8, kv=8, window=64, sinks=2, buckets=32, reach=128, seqs=3),
    _case(257, heads=3, kv=3, dh=96, buckets=24, reach=200), _case(300, heads=4, kv=2, window=1, sinks=0),
    _case(320, dh=128, window=128, sinks=4), _case(513, heads=2, kv=1, window=256, sinks=16, buckets=5, reach=1000, seqs=1),
    _case(700, heads=7, kv=1, dh=64, window=90, sinks=5, seqs=1), _case(1030, heads=1, kv=1, dh=128, buckets=64, reach=700, seqs=1),
    _case(640, heads=2, kv=2, dh=64, window=70, sinks=300, seqs=1), _case(90, heads=2, kv=1, dh=20, window=30, sinks=2, buckets=7, reach=9),
    _case(70, heads=2, kv=2, dh=7, window=12, buckets=128, reach=65), _case(130, heads=2, kv=2, dh=256, window=50, sinks=1),
    _case(130, heads=1, kv=1, dh=200, buckets=16, reach=50), _case(77, heads=3, kv=1, dh=136, window=20, sinks=20, buckets=3, reach=70),
    _case(400, heads=2, kv=2, dh=8, window=130, sinks=2, buckets=2, reach=1 << 20, seqs=1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "-".join(str(v) for v in list(c.values())[:-1]))
def test_against_fp64(case, dtype):
    c = dict(case, dtype=dtype)
    x, dy, table = _inputs(c)
    _check(_run(c, x, dy, table), _reference(c, x, dy, table))


LAUNCHES = [
    # as many sequences as fill the chip: a workgroup takes all of a key head, first keys among them
    _case(70, heads=8, kv=8, dh=16, seqs=64), _case(90, heads=8, kv=8, dh=80, window=20, sinks=2, buckets=8, reach=30, seqs=64),
    _case(70, heads=8, kv=8, dh=32, window=30, sinks=3, buckets=32, reach=64, seqs=64),
    _case(100, heads=8, kv=8, dh=128, window=40, sinks=1, seqs=40), _case(130, heads=16, kv=4, dh=64, buckets=16, reach=100, seqs=20),
    # more workgroups than the chip runs at a time, the first of them with longer walks
    _case(300, heads=16, kv=16, dh=64, window=40, sinks=1, buckets=16, reach=100, seqs=20), _case(1100, heads=8, kv=8, dh=16, window=100, sinks=3, seqs=8),
    # one long sequence: walks in parts, pairs of first keys in many chunks, first keys over several workgroups; parts that begin within a
    # query head or leave some out
    _case(1500, heads=4, kv=1, dh=16, window=64, sinks=5, buckets=12, reach=300, seqs=1),
    _case(1500, heads=4, kv=2, dh=80, window=700, sinks=70, buckets=20, reach=1000, seqs=1),
    _case(1501, heads=2, kv=1, dh=128, window=64, sinks=140, seqs=1), _case(2100, heads=6, kv=1, dh=24, window=500, buckets=9, reach=50, seqs=1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", LAUNCHES, ids=lambda c: "-".join(str(v) for v in list(c.values())[:-1]))
def test_launches_cut_up_in_every_way(case, dtype):
    c = dict(case, dtype=dtype)
    x, dy, table = _inputs(c)
    _check(_run(c, x, dy, table), _reference(c, x, dy, table))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,window,sinks,seqs", [(1500, 64, 5, 1), (70, 30, 3, 64)])
def test_a_query_that_is_not_finite_reaches_its_own_keys_only(tokens, window, sinks, seqs, dtype):
    """An infinite gradient of the last token: the first keys take it over whatever workgroup adds their distant pairs up, all others not."""
    import torch
    c = _case(tokens, heads=8, kv=8 if seqs > 1 else 2, dh=32, window=window, sinks=sinks, buckets=8, reach=40, seqs=seqs, dtype=dtype)
    x, dy, table = _inputs(c)
    clean = _run(c, x, dy, table)
    bad = dy.clone()
    bad[0, -1, ::3] = float("inf")
    got = _run(c, x, bad, table)
    at = torch.arange(tokens, device="cuda")
    key_of = (tokens - 1 - at < window) | (at < sinks)
    for k, rows in (("y", at >= 0), ("dq", at < tokens - 1), ("dk", ~key_of), ("dv", ~key_of)):
        new, old = got[k][0, rows].double(), clean[k][0, rows].double()
        assert bool(torch.isfinite(new).all()), k
        # another order of the sums: fp32 sums of at most 4 x `tokens` terms, stored with one rounding
        assert float((new - old).norm()) <= (2.0 ** -8 if dtype == "bf16" else tokens * 2.0 ** -20) * float(old.norm()), k
    assert not bool(torch.isfinite(got["dv"][0, key_of].float()).all(1).any())
    for k in ("y", "dq", "dk", "dv"):
        assert torch.equal(got[k][1:], clean[k][1:]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_micro_batches_and_repeated_calls_give_the_same_bits(dtype):
    import torch
    c = _case(150, heads=4, kv=2, dh=64, window=70, sinks=3, buckets=32, reach=128, seqs=6, dtype=dtype)
    x, dy, table = _inputs(c)
    whole = _run(c, x, dy, table)
    for n in (1, 2, 3):
        again = _run(c, x, dy, table, n=n)
        for k in whole:
            assert torch.equal(whole[k], again[k]), (n, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,window,sinks,dh", [(100, 30, 2, 64), (300, 100, 5, 128), (256, 64, 0, 64), (90, 20, 3, 20)])
def test_what_a_query_does_not_see_does_not_reach_it(tokens, window, sinks, dh, dtype):
    """Infinities and NaN in one token: rows that do not depend on it are what they are without it, up to one rounding."""
    import torch
    c = _case(tokens, heads=4, kv=2, dh=dh, window=window, sinks=sinks, buckets=8, reach=40, seqs=1, dtype=dtype)
    x, dy, table = _inputs(c)
    clean = _run(c, x, dy, table)
    h, kv = 4 * dh, 2 * dh
    at = torch.arange(tokens, device="cuda")
    for t in (tokens // 2 + 3, 0):
        sees = (at >= t) & ((at - t < window) | (t < sinks))              # queries that see token t
        key_of = (at <= t) & ((t - at < window) | (at < sinks))           # keys that token t sees
        touched = torch.zeros(tokens, dtype=torch.bool, device="cuda")    # keys that share a query with token t
        for i in torch.nonzero(sees)[:, 0].tolist():
            touched |= (at <= i) & ((i - at < window) | (at < sinks))
        for bad in (float("inf"), float("nan")):
            for where, unaffected in (("k", {"y": ~sees, "dq": ~sees, "dk": ~touched, "dv": ~touched}),
                                      ("v", {"y": ~sees, "dq": ~sees, "dk": ~touched, "dv": at >= 0}),
                                      ("dy", {"y": at >= 0, "dq": at != t, "dk": ~key_of, "dv": ~key_of})):
                a, u = x.clone(), dy.clone()
                part = {"k": a[:, t, h:h + kv], "v": a[:, t, h + kv:], "dy": u[:, t]}[where]
                part[:, ::3] = bad
                got = _run(c, a, u, table)
                for k, rows in unaffected.items():
                    new, old = got[k][:, rows].double(), clean[k][:, rows].double()
                    assert bool(torch.isfinite(new).all()), (t, bad, where, k)
                    if new.numel():
                        # another order of the sums: fp32 sums of at most `tokens` terms, stored with one rounding
                        off = float((new - old).norm()) / max(float(old.norm()), 1e-30)
                        assert off <= (2.0 ** -8 if dtype == "bf16" else tokens * 2.0 ** -22), (t, bad, where, k, off)
                hit = {"k": "y", "v": "y", "dy": "dv"}[where]
                assert not bool(torch.isfinite(got[hit].float()).all())       # and it does arrive


def test_large_scores_and_biases():
    """Scores of several hundred: the running maximum keeps the exponentials finite, one key has all the probability."""
    import torch
    for dtype in ("f32", "bf16"):
        c = _case(200, heads=2, kv=2, dh=64, window=90, sinks=2, buckets=16, reach=64, dtype=dtype)
        x, dy, table = _inputs(c)
        x[..., :128] *= 40
        table *= 300
        got = _run(c, x, dy, table)
        want = _reference(c, x.float(), dy, table)
        p_off = 2.0 ** -24 * 72 * 1.45 * 2 * float((x[..., :128].double().abs().amax() * x[..., 128:256].double().abs().amax() * 8))
        assert p_off < 0.5
        _check(got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh,tokens", [(64, 130), (20, 50)])
def test_any_address_and_rows_behind_the_last(dtype, dh, tokens):
    """Callers' tensors that start at an odd element; nothing is written outside them."""
    import torch
    c = _case(tokens, heads=2, kv=1, dh=dh, window=40, sinks=1, buckets=6, reach=20, dtype=dtype)
    x, dy, table = _inputs(c)
    st = _stage(c, _params(table))

    def odd(t, fill=None):
        flat = torch.full((t.numel() + 64,), 7.0, dtype=t.dtype, device=t.device)
        view = flat[1: 1 + t.numel()].view(t.shape)
        if fill is not None:
            view.copy_(fill)
        return flat, view

    x2, dy2 = x.reshape(c["seqs"], -1), dy.reshape(c["seqs"], -1)
    yf, y = odd(dy2)
    dxf, dx = odd(x2)
    st.forward(0, 0, odd(x2, x2)[1], y)
    st.backward(0, odd(dy2, dy2)[1], dx)
    got = _split(c, y, dx, st.grad)
    _check(got, _reference(c, x, dy, table))
    for flat, t in ((yf, y), (dxf, dx)):
        assert float(flat[0]) == 7.0 and bool((flat[1 + t.numel():] == 7.0).all())
    st.close()


def test_no_input_gradient_asked_for():
    """A first stage: the table's gradient all the same, and without a table nothing."""
    import torch
    c = _case(70, heads=2, kv=2, window=20, sinks=1, buckets=8, reach=30)
    x, dy, table = _inputs(c)
    st = _stage(c, _params(table), needs_dx=False)
    st.forward(0, 0, x.reshape(2, -1))
    st.backward(0, dy.reshape(2, -1))
    assert torch.equal(st.grad[:16].view(2, 8), _run(c, x, dy, table)["dtable"])
    st.close()
    c = dict(c, buckets=0, reach=0)
    st = _stage(c, [], needs_dx=False)
    st.forward(0, 0, x.reshape(2, -1))
    st.backward(0, dy.reshape(2, -1))
    assert st.blend_update(0) == 1
    st.close()


def test_gradients_against_differences():
    """The loss sum(y * dy) in fp32, moved along random directions of the inputs and of the table."""
    import torch
    c = _case(60, heads=4, kv=2, dh=32, window=25, sinks=2, buckets=8, reach=40, dtype="f32")
    x, dy, table = _inputs(c)
    got = _run(c, x, dy, table)
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    dx = torch.cat([got["dq"], got["dk"], got["dv"]], 2).double()
    loss = lambda x, t: float((_run(c, x, dy, t)["y"].double() * dy.double()).sum())
    eps = 2.0 ** -7
    for d in range(4):
        along = torch.randn(x.shape, generator=g, device="cuda")
        bias = torch.randn(table.shape, generator=g, device="cuda")
        for a, b, want in ((along, 0 * bias, float((dx * along.double()).sum())), (0 * along, bias, float((got["dtable"].double() * bias.double()).sum()))):
            diff = (loss(x + eps * a, table + eps * b) - loss(x - eps * a, table - eps * b)) / (2 * eps)
            # third-order term of the difference and the rounding of y: directions have about |dx| sqrt(values) of slope
            slope = float(dx.norm()) if a.abs().sum() > 0 else float(got["dtable"].double().norm())
            assert abs(diff - want) <= 2e-2 * max(abs(want), slope), (d, diff, want)


def test_update_and_versions_follow_the_oracle():
    """A decoder block with this layer, with staleness, under every policy."""
    from stage_parity import run_stage
    from synth_inputs import workloads as W
    for dtype, dh in (("f32", 16), ("bf16", 64)):
        d = 4 * dh
        specs = W.windowed_block(d, 4, 2 * d, 50, 2, 20, 2, 8, 30)
        for policy in ("convex", "latest", "stashed", "eq1"):
            print(dtype, policy, run_stage(specs, f"local_{dtype}", dtype, mb=2, n=2, policy=policy))


def test_last_layer_of_a_stage():
    from stage_parity import run_stage
    from synth_inputs import workloads as W
    for dtype in ("f32", "bf16"):
        specs = (W.Dense(32, 256, "none", tokens=70), W.LocalAttention(128, 2, 70, 1, 33, 2, 6, 20))
        print(dtype, run_stage(specs, f"local_last_{dtype}", dtype, mb=2, n=2))


def test_layers_beside_it():
    """First in a stage, one behind another, behind a ReLU, in front of a residual begin and of the addition itself."""
    from stage_parity import run_stage
    from synth_inputs import workloads as W
    for dtype in ("f32", "bf16"):
        specs = (W.LocalAttention(96, 6, 45, 2, 20, 1, 4, 9), W.LocalAttention(64, 4, 45, 1), W.Residual(64, 45, "begin"),
                 W.Dense(64, 96, "relu", tokens=45), W.LocalAttention(64, 4, 45, 1, 9, 0, 8, 30), W.Residual(64, 45, "add"),
                 W.Dense(64, 40, "gelu", tokens=45))
        print(dtype, run_stage(specs, f"local_beside_{dtype}", dtype, mb=2, n=2, policy="convex"))


def test_forward_streams():
    """Micro-batches on streams of their own share no scratch memory: the same bits."""
    import torch
    c = _case(120, heads=4, kv=2, dh=64, window=50, sinks=3, buckets=32, reach=128, seqs=6)
    x, dy, table = _inputs(c)
    want = _run(c, x, dy, table, n=3)
    for streams in (1, 3):
        st = _stage(c, _params(table), n=3, forward_stream=streams)
        y = torch.empty(6, st.out_elems, dtype=st.tdtype, device="cuda")
        torch.cuda.synchronize()
        for j in range(3):
            for ub in range(3):
                st.forward(j, ub, x.reshape(6, -1)[2 * ub: 2 * ub + 2], y[2 * ub: 2 * ub + 2])
            st.forward_join()
            dx, _ = st.backward(j, dy.reshape(6, -1))
            got = _split(c, y, dx, st.grad)
            for k in want:
                assert torch.equal(got[k], want[k]), (streams, j, k)
            st.blend_update(j)
        st.close()


def test_captured_into_a_graph_and_replayed():
    """Forward, backward and update in one graph, replayed on new inputs between eager work; two stages captured one after the
    other have workspaces of their own."""
    import torch
    cases = [_case(140, heads=4, kv=2, dh=64, window=60, sinks=3, buckets=32, reach=128), _case(65, heads=2, kv=2, dh=128, window=30, seqs=3)]
    stream = torch.cuda.Stream()
    graphs = []
    for c in cases:
        x, dy, table = _inputs(c)
        st = _stage(c, _params(table), stream=stream)
        xs, ds = x.reshape(c["seqs"], -1).clone(), dy.reshape(c["seqs"], -1).clone()
        y, dx = torch.empty_like(ds), torch.empty_like(xs)

        def step(j):
            st.forward(j, 0, xs, y)
            st.backward(j, ds, dx)
            st.blend_update(j)

        torch.cuda.synchronize()
        step(0)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(1)
        graphs.append((c, st, graph, xs, ds, y, dx, table))
    for seed in range(4):
        todo = []
        for c, st, graph, xs, ds, y, dx, table in graphs:
            x, dy, _ = _inputs(c, seed=10 * seed + 5)
            xs.copy_(x.reshape(xs.shape))
            ds.copy_(dy.reshape(ds.shape))
            todo.append((x, dy))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for g in graphs:
                g[2].replay()
        torch.cuda.synchronize()
        for (c, st, graph, xs, ds, y, dx, table), (x, dy) in zip(graphs, todo):
            want = _run(c, x, dy, table)
            got = _split(c, y, dx, st.grad)
            for k in want:
                assert torch.equal(got[k], want[k]), (seed, k)
    for g in graphs:
        g[1].close()


def test_two_stages_on_two_streams():
    import torch
    c = _case(256, heads=4, kv=2, dh=64, window=100, sinks=3, buckets=32, reach=128, seqs=4)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    work, want = [], []
    for i, s in enumerate(streams):
        x, dy, table = _inputs(c, seed=100 + i)
        want.append(_run(c, x, dy, table))
        work.append((_stage(c, _params(table), stream=s), x.reshape(4, -1), dy.reshape(4, -1), torch.empty(4, 256 * 256, dtype=x.dtype, device="cuda"),
                     torch.empty_like(x.reshape(4, -1))))
    torch.cuda.synchronize()
    for j in range(3):
        for st, x, dy, y, dx in work:
            st.forward(j, 0, x, y)
        for st, x, dy, y, dx in work:
            st.backward(j, dy, dx)
            st.blend_update(j)
    torch.cuda.synchronize()
    for (st, x, dy, y, dx), w in zip(work, want):
        got = _split(c, y, dx, st.grad)
        for k in w:
            assert torch.equal(got[k], w[k]), k
        st.close()


def test_buckets_without_pairs_get_no_gradient():
    import torch
    c = _case(20, heads=2, kv=2, dh=64, window=6, sinks=0, buckets=128, reach=4000)
    x, dy, table = _inputs(c)
    got = _run(c, x, dy, table)["dtable"]
    assert bool((got[:, 6:] == 0).all()) and bool((got[:, :6] != 0).all())
