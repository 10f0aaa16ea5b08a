"""The position bias of windowed attention where a query or a table entry is not finite: only what a visible pair has in common with it changes.

Buckets of other pairs are held to what they are without it.  Not to the same bits: the rows of a wave move the references of their exponentials
together, so that an infinite score moves its neighbours' too, and their exponentials are rounded otherwise.  Both runs lie within the bound of
test_gpu_local_attention.py around the exact sums, so they differ by twice that at most; a bucket without a visible pair has a bound of zero."""
import numpy as np
import pytest

from test_gpu_local_attention import _reference

pytestmark = pytest.mark.gpu


def _run(c, x, dy, table, odd=False):
    """y, dx and dtable of one stage of this layer; odd: tensors that start at an odd element, which other kernels take."""
    import torch
    from paper_2509_23241_amd.runner import GpuStage
    layer = ("local", c["heads"] * c["dh"], c["heads"], c["tokens"], c["kv"], c["window"], c["sinks"], c["buckets"], c["reach"])
    st = GpuStage([layer], [table.cpu().numpy(), np.zeros(0, np.float32)], dtype=c["dtype"], mb=x.shape[0], n=1, stage_index=1, num_stages=2,
                  policy="latest", lam=0.1, lr=0.0, momentum=0.0)
    put = lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape[0], -1) if odd else t.reshape(t.shape[0], -1)
    y = put(torch.zeros_like(dy))
    st.forward(0, 0, put(x), y)
    dx = put(torch.zeros_like(x))
    st.backward(0, put(dy), dx)
    out = {"y": y.view(dy.shape).clone(), "dx": dx.view(x.shape).clone(), "dtable": st.grad[: table.numel()].view_as(table).clone()}
    st.close()
    return out


def _inputs(c, seqs=1):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(c["tokens"] + c["window"])
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    x = torch.randn(seqs, c["tokens"], (c["heads"] + 2 * c["kv"]) * c["dh"], generator=g, device="cuda").to(t)
    dy = torch.randn(seqs, c["tokens"], c["heads"] * c["dh"], generator=g, device="cuda").to(t)
    return x, dy, torch.randn(c["heads"], c["buckets"], generator=g, device="cuda")


CASES = [dict(tokens=150, heads=4, kv=2, dh=64, window=6, sinks=0, buckets=32, reach=128),
         dict(tokens=300, heads=2, kv=2, dh=128, window=40, sinks=2, buckets=24, reach=200),
         dict(tokens=700, heads=2, kv=1, dh=32, window=250, sinks=2, buckets=64, reach=600),
         dict(tokens=700, heads=2, kv=2, dh=128, window=260, sinks=0, buckets=64, reach=600),
         dict(tokens=90, heads=2, kv=1, dh=20, window=12, sinks=1, buckets=16, reach=60)]
ids = lambda c: "-".join(str(v) for v in c.values())


def _pairs(c, i):
    """Distances of the keys that query i sees."""
    return [i - j for j in range(i + 1) if i - j < c["window"] or j < c["sinks"]]


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_a_query_reaches_the_buckets_of_its_pairs_only(case, dtype, odd):
    import torch
    from oracle.layers import distance_buckets
    c = dict(case, dtype=dtype)
    x, dy, table = _inputs(c)
    bucket = distance_buckets(c["tokens"], c["buckets"], c["reach"])
    clean = _run(c, x, dy, table, odd)
    apart = 2 * _reference(c, x, dy, table)["dtable"][1]
    for i in (c["tokens"] - 1, c["tokens"] // 2 + 5, 9):
        hit = np.zeros(c["buckets"], bool)
        hit[bucket[_pairs(c, i)]] = True
        hit = torch.from_numpy(hit).cuda()
        for where in ("dy", "q"):
            for bad in (np.inf, np.nan):
                a, u = x.clone(), dy.clone()
                if where == "dy":
                    u[0, i, ::3] = bad
                else:
                    a[0, i, : c["heads"] * c["dh"]: 3] = bad
                got = _run(c, a, u, table, odd)["dtable"]
                off = (got.double() - clean["dtable"].double()).abs()
                assert bool((off <= apart)[:, ~hit].all()), (i, where, bad)
                assert not bool(torch.isfinite(got).all()), (i, where, bad)


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [c for c in CASES if c["sinks"] == 0] + [dict(tokens=500, heads=2, kv=2, dh=64, window=200, sinks=0, buckets=16, reach=400)], ids=ids)
def test_entries_that_no_visible_pair_has(case, dtype, odd):
    """Entries of distances beyond the window hold anything: same bits everywhere, and a gradient of 0 for them."""
    import torch
    from oracle.layers import distance_buckets
    c = dict(case, dtype=dtype)
    x, dy, table = _inputs(c, seqs=2)
    used = int(distance_buckets(c["tokens"], c["buckets"], c["reach"])[c["window"] - 1]) + 1
    assert used < c["buckets"]
    clean = _run(c, x, dy, table, odd)
    assert bool((clean["dtable"][:, used:] == 0).all()) and all(bool(torch.isfinite(t).all()) for t in clean.values())
    for value in (np.nan, np.inf, -np.inf, 3e38):
        other = table.clone()
        other[:, used:] = value
        got = _run(c, x, dy, other, odd)
        for k in clean:
            assert torch.equal(got[k], clean[k]), (value, k)
