"""The operators of a decoder stage that is tuned on preferences and rewards, as they are used together: rotary positions in front of
attention on shared key heads, gated feed-forward halves, log probabilities, both losses; over steps, on streams, in graphs."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
T, D, HEADS, KV, DH, INNER, CLASSES = 24, 64, 4, 2, 16, 88, 50


def _specs():
    from synth_inputs import workloads as W
    res = lambda mark: W.Residual(D, T, mark)
    half = (res("begin"), W.LayerNorm(D, T), W.Dense(D, (HEADS + 2 * KV) * DH, "none", tokens=T), W.Rotary(HEADS, KV, DH, T, DH, "halves"),
            W.LocalAttention(HEADS * DH, HEADS, T, KV, 0, 0), W.Dense(HEADS * DH, D, "none", tokens=T), res("add"))
    other = (res("begin"), W.LayerNorm(D, T), W.Gated(D, INNER, "silu", T), W.Dense(INNER, D, "none", tokens=T), res("add"))
    return half + other + (W.LayerNorm(D, T), W.Dense(D, CLASSES, "none", tokens=T))


def _params(specs, dtype):
    from synth_inputs import workloads as W
    rng = np.random.default_rng(11)
    out = []
    for s in specs:
        if not s.param_shapes():
            continue
        a, b = s.param_shapes()
        out.append(np.ones(a) if s.kind == "ln" else rng.standard_normal(a) / np.sqrt(a[1]))
        out.append(0.1 * rng.standard_normal(b))
    return [W.round_bf16(p) if dtype == "bf16" else W.round_f32(p) for p in out]


def _make(dtype, mb, n, lr=0.0, device="cuda:0", **more):
    from paper_2509_23241_amd.runner import GpuStage, layer_tuple
    specs = _specs()
    params = _params(specs, dtype)
    more = {"policy": "latest", **more}
    st = GpuStage([layer_tuple(s) for s in specs], params, dtype=dtype, mb=mb, n=n, stage_index=1, num_stages=2, lam=0.1, lr=lr, momentum=0.5,
                  device=device, **more)
    return st, specs, params


def _batch(dtype, samples, seed, device="cuda:0"):
    import torch
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows = samples * T
    x = torch.randn(samples, T * D, generator=g).to(t)
    ids = torch.randint(0, CLASSES, (rows,), generator=g, dtype=torch.int32)
    ids[torch.rand(rows, generator=g) < 0.3] = -1
    adv = torch.randn(rows, generator=g)
    return [v.to(device) for v in (x, ids, adv)]


def _forward(st, j, x):
    import torch
    y = torch.empty(x.shape[0], st.out_elems, dtype=st.tdtype, device=st.device)
    for ub in range(st.n):
        st.forward(j, ub, x[ub * st.mb:(ub + 1) * st.mb], y[ub * st.mb:(ub + 1) * st.mb])
    st.forward_join()
    return y


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("policy", ["latest", "convex"])
def test_steps_of_both_losses_follow_the_oracle(policy, dtype):
    """Log probabilities of the first weights as the reference and the old policy, then steps of either loss: losses, gradients and new
    weights against the oracle's stage and losses, to the tolerances of the other stages (1e-4 and 2e-2 of a tensor's norm)."""
    import torch
    from oracle import layers as OL
    from oracle.stage import Stage
    from parity_utils import TOL, oracle_flat_to_arena, rel_err, to_np
    from synth_inputs import workloads as W
    tol = TOL[dtype]
    mb, n = 2, 2
    st, specs, params = _make(dtype, mb, n, lr=0.5, policy=policy)
    ost = Stage(specs, params, policy=policy, lam=0.1, lr=0.5, momentum=0.5, n=n, storage=W.round_bf16 if dtype == "bf16" else None)
    for j, kind in enumerate(("policy", "preference", "policy", "preference")):
        x, ids, adv = _batch(dtype, mb * n, j)
        xr = x.double().cpu().numpy().reshape(mb * n, T, D)
        logits = _forward(st, j, x)
        want = np.concatenate([ost.forward(j, ub, xr[ub * mb:(ub + 1) * mb]) for ub in range(n)]).reshape(-1, CLASSES)
        assert rel_err(to_np(logits), want) < tol
        z, idn = to_np(logits).astype(np.float64).reshape(-1, CLASSES), ids.cpu().numpy()
        old = st.logprobs(logits, ids)
        assert rel_err(to_np(old), OL.policy_loss(z, idn, np.zeros(len(z)), np.zeros(len(z)))[2]) < 1e-5
        if kind == "policy":
            behind = old - 0.1
            loss, dy, logp = st.loss_policy(j, logits, ids, behind, adv, ref_logp=old + 0.2, kl_weight=0.1, clip_high=0.3)
            ref = OL.policy_loss(z, idn, to_np(behind), to_np(adv), None, to_np(old + 0.2), 0.2, 0.3, 0.1)
        else:
            sums = torch.where(ids >= 0, old, 0).view(mb * n, T).sum(1) + torch.tensor([-1.0, 1.0] * (mb * n // 2), device="cuda")
            loss, dy, logp = st.loss_preference(j, logits, ids, sums, beta=0.5, label_smoothing=0.1)
            ref = OL.preference_loss(z, idn, to_np(sums), T, None, 0.5, 0.1)
        assert torch.equal(torch.where(ids >= 0, logp, 0.0), torch.where(ids >= 0, old, 0.0))
        assert abs(float(loss) - ref[0]) < 1e-4 * (1 + abs(ref[0])) and rel_err(to_np(dy).reshape(-1, CLASSES), ref[1]) < (1e-4 if dtype == "f32" else 2e-2)
        dx, delta = st.backward(j, dy)
        dxr = ost.backward(j, to_np(dy).astype(np.float64).reshape(mb * n, T, CLASSES))
        assert rel_err(to_np(dx), dxr.reshape(mb * n, -1)) < tol and rel_err(to_np(st.grad)[: st.P], oracle_flat_to_arena(st, ost.flat(ost.g))) < tol
        st.blend_update(j)
        ost.update(j)
        assert rel_err(to_np(st.export(ost.latest)), oracle_flat_to_arena(st, ost.flat(ost.weights[ost.latest]))) < tol
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_micro_batches_on_streams_and_in_one_call_give_the_same_bits(dtype):
    import torch
    x, ids, adv = _batch(dtype, 6, 3)

    def step(**more):
        st, _, _ = _make(dtype, 2, 3, **more)
        logits = _forward(st, 0, x)
        loss, dy, logp = st.loss_policy(0, logits, ids, torch.zeros_like(adv) - 4, adv)
        dx, _ = st.backward(0, dy)
        out = [t.clone() for t in (logits, loss, dy, logp, dx, st.grad)]
        st.close()
        return out
    one = step()
    for streams in (1, 3):
        for a, b in zip(one, step(forward_stream=streams)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_into_a_graph_and_replayed(dtype):
    """Forward, loss, backward and update in one graph for either loss, replayed on new inputs between eager work; two stages captured one
    after the other have workspaces of their own."""
    import torch
    stream = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(stream):
        for kind in ("policy", "preference"):
            st, _, _ = _make(dtype, 4, 1, stream=stream, ring_capacity=1, max_in_flight=1)
            x, ids, adv = _batch(dtype, 4, 20)
            ref = torch.full((4,), -60.0, device="cuda")
            bufs = dict(y=torch.empty(4, st.out_elems, dtype=st.tdtype, device="cuda"), dx=torch.empty_like(x))

            def step(j, st=st, kind=kind, x=x, ids=ids, adv=adv, ref=ref, bufs=bufs):
                st.forward(j, 0, x, bufs["y"])
                if kind == "policy":
                    out = st.loss_policy(j, bufs["y"], ids, adv - 4, adv, kl_weight=0.1, ref_logp=adv - 3)
                else:
                    out = st.loss_preference(j, bufs["y"], ids, ref)
                st.backward(j, out[1], bufs["dx"])
                st.blend_update(j)
                return out
            step(0)
            graph = torch.cuda.CUDAGraph()
            stream.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                out = step(1)
            graphs.append((st, graph, out, bufs, x, ids, adv, step))
        for k in range(4):
            for st, graph, out, bufs, x, ids, adv, step in graphs:
                for t, v in zip((x, ids, adv), _batch(dtype, 4, 30 + k)):
                    t.copy_(v)
                graph.replay()
            stream.synchronize()
            for i, (st, graph, out, bufs, x, ids, adv, step) in enumerate(graphs):
                got = [t.clone() for t in out] + [bufs["y"].clone(), bufs["dx"].clone(), st.grad.clone()]
                want = step(100 + k)
                for a, b in zip(got, list(want) + [bufs["y"], bufs["dx"], st.grad]):
                    assert torch.equal(a, b), (k, i)
            stream.synchronize()
    for st, *_ in graphs:
        st.close()


def test_two_stages_on_streams_of_their_own():
    """Work of one stage beside that of another: no scratch memory is shared, results are those of one after the other."""
    import torch
    alone = []
    for seed in (1, 2):
        st, _, _ = _make("bf16", 4, 1)
        x, ids, adv = _batch("bf16", 4, seed)
        y = _forward(st, 0, x)
        out = st.loss_preference(0, y, ids, torch.zeros(4, device="cuda"))
        dx, _ = st.backward(0, out[1])
        alone.append([t.clone() for t in (*out, dx, st.grad)])
        st.close()
    streams = [torch.cuda.Stream() for _ in range(2)]
    stages = [_make("bf16", 4, 1, stream=s)[0] for s in streams]
    data = [_batch("bf16", 4, seed) for seed in (1, 2)]
    ref = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        j = int(stages[0].query().latest_version)
        got = []
        for st, s, (x, ids, adv) in zip(stages, streams, data):
            with torch.cuda.stream(s):
                y = _forward(st, j, x)
                out = st.loss_preference(j, y, ids, ref)
                dx, _ = st.backward(j, out[1])
                got.append([*out, dx])
        torch.cuda.synchronize()
        for st, g, want in zip(stages, got, alone):
            for a, b in zip(g + [st.grad], want):
                assert torch.equal(a, b)
            st.blend_update(j)
        torch.cuda.synchronize()
    for st in stages:
        st.close()
