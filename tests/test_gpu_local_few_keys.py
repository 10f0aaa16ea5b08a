"""dQ of windowed attention for queries that see at most 32 keys, where all values have a large part in common.

delta = dy.y then is much larger than the dP - delta that it is taken from, and what rounds the stored y to bf16 (2^-8 of it) is larger than dS:
queries of few keys must not have it in their dq.  Bounds as in test_gpu_local_attention.py without that term: unit f = 2^-24, over the K keys
that a query sees
  p        2 (dh + 8) f log2(e) (largest score + 1) + (K + 8) f of itself
  dP       (dh + 8) f sum |dy||v|
  delta    sum over p of what p and dP are off, (K + 8) f sum p |dP|
  dS       p times (what dP and delta are off + |dP - delta| times what p is off), 2^-8 where it enters the product in bf16
  dq       (K + 8) f of the sum, 2^-8 of the stored value."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
F = 2.0 ** -24


def _dq(c, x, dy, table, odd):
    import torch
    from paper_2509_23241_amd.runner import GpuStage
    layer = ("local", c["heads"] * c["dh"], c["heads"], c["tokens"], c["kv"], c["window"], c["sinks"], c["buckets"], c["reach"])
    params = [] if table is None else [table.cpu().numpy(), np.zeros(0, np.float32)]
    st = GpuStage([layer], params, dtype=c["dtype"], mb=x.shape[0], n=1, stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0)
    put = lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape[0], -1) if odd else t.reshape(t.shape[0], -1)
    st.forward(0, 0, put(x))
    dx = put(torch.zeros_like(x))
    st.backward(0, put(dy), dx)
    out = dx.view(x.shape)[..., : c["heads"] * c["dh"]].clone()
    st.close()
    return out


def _check(c, odd=False, common=64.0):
    import torch
    from oracle.layers import distance_buckets
    h, kv, dh, S, n = c["heads"], c["kv"], c["dh"], c["tokens"], c.get("seqs", 2)
    g = torch.Generator(device="cuda")
    g.manual_seed(S + dh)
    t, u = (torch.bfloat16, 2.0 ** -8) if c["dtype"] == "bf16" else (torch.float32, F)
    x = torch.randn(n, S, h + 2 * kv, dh, generator=g, device="cuda")
    x[:, :, h + kv:] += common
    x = x.to(t)
    dy = (torch.randn(n, S, h, dh, generator=g, device="cuda") + 0.5).to(t)
    table = torch.randn(h, c["buckets"], generator=g, device="cuda") if c["buckets"] else None
    got = _dq(c, x.view(n, S, -1), dy.view(n, S, -1), table, odd).view(n, S, h, dh).double()
    spread = torch.arange(kv, device="cuda").repeat_interleave(h // kv)
    x, dy = x.double(), dy.double()
    at = torch.arange(S, device="cuda")
    worst, rows = 0.0, 0
    for i in range(S):
        keys = at[(at <= i) & ((i - at < (c["window"] or S)) | (at < c["sinks"]))]
        K = len(keys)
        if K > 32:
            continue
        rows += 1
        q, k, v, do = x[:, i, :h], x[:, keys][:, :, h + spread], x[:, keys][:, :, h + kv + spread], dy[:, i]      # [n, h, dh], [n, K, h, dh]
        s = (q[:, None] * k).sum(3) / math.sqrt(dh)
        size = (q[:, None] * k).abs().sum(3) / math.sqrt(dh)
        if table is not None:
            b = table.double()[:, torch.from_numpy(distance_buckets(S, c["buckets"], c["reach"])).cuda()[i - keys]].t()
            s, size = s + b, size + b.abs()
        p = s.softmax(1)
        ep = p * (2 * (dh + 8) * F * 1.4427 * (float(size.max()) + 1) + (K + 8) * F)
        dp, adp = (do[:, None] * v).sum(3), (do[:, None] * v).abs().sum(3)
        edp = (dh + 8) * F * adp
        delta = (p * dp).sum(1, keepdim=True)
        edelta = (ep * dp.abs() + p * edp).sum(1, keepdim=True) + (K + 8) * F * (p * dp.abs()).sum(1, keepdim=True)
        ds = p * (dp - delta)
        eds = ep * (dp - delta).abs() + p * (edp + edelta)
        eds = eds + ((u if c["dtype"] == "bf16" else 0) + (K + 8) * F) * (ds.abs() + eds)
        dq = (ds[..., None] * k).sum(1) / math.sqrt(dh)
        bound = (eds[..., None] * k.abs()).sum(1) / math.sqrt(dh)
        bound = bound + u * (dq.abs() + bound)
        worst = max(worst, float(((got[:, i] - dq).abs() / (bound + 1e-30)).max()))
    print(rows, "rows, share of the bound %.3g" % worst)
    assert rows and worst <= 1.0, worst


def _case(tokens, heads=2, dh=64, kv=2, window=0, sinks=0, buckets=0, reach=0, **more):
    return dict(tokens=tokens, heads=heads, dh=dh, kv=kv, window=window, sinks=sinks, buckets=buckets, reach=reach, **more)


CASES = [_case(1), _case(20, dh=128), _case(33), _case(33, dh=128, heads=4, kv=1), _case(64, heads=3, kv=1, dh=80), _case(65, buckets=8, reach=30),
         _case(200, heads=8, kv=8, dh=64, window=64, sinks=2, buckets=32, reach=128, seqs=12), _case(200, window=31, sinks=1, heads=4, kv=2),
         _case(130, window=8, sinks=0, dh=128), _case(130, window=16, sinks=16, buckets=16, reach=100), _case(70, heads=16, kv=1, dh=32, window=3),
         _case(1024, dh=128), _case(1024, window=256, sinks=4, buckets=24, reach=300), _case(300, window=20, sinks=2, heads=7, kv=1, dh=128),
         _case(150, heads=16, kv=16, window=20, sinks=2, seqs=40)]
ids = lambda c: "-".join(str(v) for v in c.values())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_queries_of_few_keys(case, dtype):
    _check(dict(case, dtype=dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [_case(1, dh=20), _case(33, dh=20), _case(40, dh=200), _case(90, dh=256, window=20, sinks=2, buckets=8, reach=30),
                                  _case(130, heads=4, kv=2, dh=7, window=9), _case(300, heads=3, kv=1, dh=136, window=60, sinks=1)], ids=ids)
def test_queries_of_few_keys_in_other_heads(case, dtype):
    _check(dict(case, dtype=dtype))


@pytest.mark.parametrize("case", [_case(33), _case(200, heads=4, kv=2, dh=128, window=12, sinks=3, buckets=8, reach=30), _case(150, window=90)], ids=ids)
def test_queries_of_few_keys_at_any_address(case):
    _check(dict(case, dtype="bf16"), odd=True)
