"""Operators of a decoder stage that learns from a stored teacher, as timed cases: each in a plain form of elementary torch
operations (`own` false) and through the library's stages (`own` true).

  local    causal attention over the last `window` keys (0: all) and the first `sinks` keys, `heads` query heads on `kv_heads`
           key heads, forward and backward: a stage of one such layer, its forward pass, backward pass and update (learning
           rate 0, so that passes on one state repeat)
  bias     the same with a learned bias per head and distance bucket on the scores, whose gradient is returned too
  distill  the loss at a last stage that learns from a teacher's `k` stored top logits and from labels, with its gradient

The ranges (`draw`), on which the listed cases are points:
  local, bias  1 .. 64 sequences of 1 .. 8192 tokens, heads 32 .. 128 wide, 1 .. 16 of them, key heads that divide them, windows
               from 1 key to all, 0 .. 64 sinks, 4 .. 64 buckets up to distance 1024; bf16, and fp32 at a sixteenth of the work
  distill      1 .. 16384 rows of 10 .. 64000 classes, 1 .. 256 stored logits a row (some rows with fewer, some with none),
               temperatures 1 .. 4, labels weighted 0 .. 1; bf16 and fp32
"""
import math

import torch

DEVICE = "cuda:0"
own = False  # set by whoever imports the file


# ---- the cases -----------------------------------------------------------------------------------------------------

def _attention(seqs, tokens, heads, head, kv_heads, window, sinks, dtype, buckets=0, max_distance=0):
    return dict(kind="bias" if buckets else "local", seqs=seqs, tokens=tokens, heads=heads, head=head, kv_heads=kv_heads,
                window=window, sinks=sinks, buckets=buckets, max_distance=max_distance, dtype=dtype)


def _distill(rows, classes, k, temperature, label_weight, dtype):
    return dict(kind="distill", rows=rows, classes=classes, k=k, temperature=temperature, label_weight=label_weight, dtype=dtype)


def listed():
    return [
        # the smallest call: one short sequence, where launches decide
        dict(_attention(1, 16, 4, 64, 4, 8, 2, "bf16"), name="local_bf16_16"),
        # a decoder at the size of the transformer configuration (8 sequences of 1024 tokens, 16 heads of 128)
        dict(_attention(8, 1024, 16, 128, 16, 256, 4, "bf16"), name="local_bf16_1024"),
        # one long document, four query heads to a key head
        dict(_attention(1, 16384, 8, 128, 2, 1024, 16, "bf16"), name="local_bf16_16384"),
        # single precision, as the smallest configuration trains
        dict(_attention(4, 512, 8, 64, 8, 128, 1, "f32"), name="local_f32_512"),
        # a small model in single precision on sequences that fill no tile
        dict(_attention(2, 50, 4, 32, 4, 0, 0, "f32", 16, 64), name="bias_f32_50"),
        # the transformer configuration's attention over all earlier tokens, 32 buckets up to distance 128
        dict(_attention(8, 1024, 16, 128, 16, 0, 0, "bf16", 32, 128), name="bias_bf16_1024"),
        # a small decoder on short sequences of odd length, window and bias together
        dict(_attention(32, 200, 8, 64, 8, 64, 2, "bf16", 32, 128), name="bias_bf16_200"),
        # heads of another width, shared key heads, buckets that reach far
        dict(_attention(4, 777, 6, 80, 2, 300, 3, "bf16", 24, 512), name="bias_bf16_777"),
        # the smallest classifier: 32 rows of 10 classes
        dict(_distill(32, 10, 3, 2.0, 0.5, "f32"), name="distill_f32_10"),
        # a last stage with 1000 classes
        dict(_distill(2048, 1000, 10, 2.0, 0.5, "bf16"), name="distill_bf16_1000"),
        # the decoder's vocabulary, one micro-batch of 8 x 1024 tokens
        dict(_distill(8192, 32000, 64, 2.0, 0.25, "bf16"), name="distill_bf16_32000"),
        # an odd number of classes and of rows in single precision, the teacher alone
        dict(_distill(1003, 32003, 33, 3.0, 0.0, "f32"), name="distill_f32_32003"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _int(rng, lo, hi):
    return min(hi, max(lo, int(round(_log(rng, lo, hi)))))


def _draw_once(rng):
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if rng.random() < 1 / 3:
        classes, k = _int(rng, 10, 64000), _int(rng, 1, 256)
        if rng.random() < 0.5:
            classes = max(16, classes // 8 * 8)
        return _distill(_int(rng, 1, 16384), classes, min(k, classes), rng.choice([1.0, 1.5, 2.0, 4.0]),
                        rng.choice([0.0, 0.25, 0.5, 1.0]), dtype)
    tokens = _int(rng, 1, 8192)
    if rng.random() < 0.5:
        tokens = max(64, tokens // 64 * 64)
    kv_heads, group = rng.choice([(1, 1), (2, 1), (4, 1), (8, 1), (16, 1), (1, 4), (2, 4), (4, 2), (3, 2), (1, 7)])
    window = rng.choice([0, _int(rng, 1, tokens), _int(rng, 1, tokens)])
    sinks = rng.choice([0, 1, 4, _int(rng, 1, 64)]) if window else 0
    buckets, reach = 0, 0
    if rng.random() < 0.5:
        buckets, reach = rng.choice([(32, 128), (rng.randint(4, 64), _int(rng, 64, 1024))])
    return _attention(_int(rng, 1, 64), tokens, kv_heads * group, rng.choice([32, 64, 64, 80, 96, 128, 128]), kv_heads, window,
                      sinks, dtype, buckets, reach)


def draw(rng):
    """Sizes are redrawn until the case costs no more than the largest listed one: the scores that the plain form keeps whole
    and the operations for attention (fp32 leaves a sixteenth of them), the logits for the loss."""
    while True:
        c = _draw_once(rng)
        if c["kind"] == "distill":
            if c["rows"] * c["classes"] * (1 if c["dtype"] == "bf16" else 2) <= 8192 * 32000:
                return c
        elif c["seqs"] * c["heads"] * c["tokens"] ** 2 <= 8 * 16384 ** 2 // (1 if c["dtype"] == "bf16" else 16) and \
                work(c)["flops"] <= 1.2e11 / (1 if c["dtype"] == "bf16" else 16):
            return c


# ---- what a pass has to do -------------------------------------------------------------------------------------------

def _pairs(c):
    """Visible (query, key) pairs of one sequence and head."""
    t, w, s = c["tokens"], c["window"] or c["tokens"], c["sinks"]
    return sum(min(i + 1, w) + min(s, max(0, i + 1 - w)) for i in range(t))


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "distill":
        # logits in, their gradient out, stored logits and classes in; two exponentials and some sums a logit
        return {"bytes": c["rows"] * (2 * c["classes"] * es + 8 * c["k"] + 4), "flops": 10 * c["rows"] * c["classes"]}
    q, kv = c["heads"] * c["head"], 2 * c["kv_heads"] * c["head"]
    # queries, keys, values in and their gradients out; the output out, its gradient in; two products forward, five backward
    return {"bytes": c["seqs"] * c["tokens"] * es * (2 * (q + kv) + 2 * q) + 8 * c["heads"] * c["buckets"],
            "flops": 14 * c["head"] * c["heads"] * c["seqs"] * _pairs(c)}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _first_distances(buckets, max_distance):
    """The first distance of each bucket: distances 0 .. half - 1 have one each, the others grow by equal ratios up to
    max_distance.  Bucket half + t starts at the smallest whole d with d^n >= half^(n - t) max_distance^t, n = buckets - half."""
    half = buckets // 2
    n = buckets - half
    first = list(range(half))
    for t in range(n):
        limit = half ** (n - t) * max_distance ** t
        d = max(half, int(half * (max_distance / half) ** (t / n)) - 2)
        while d ** n < limit:
            d += 1
        first.append(d)
    return first


def _inputs(c, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE)

    s = {"case": c}
    if c["kind"] == "distill":
        rows, classes, k = c["rows"], c["classes"], c["k"]
        logits = 3 * normal(rows, classes)
        s["logits"] = logits.to(_type(c))
        logits.mul_(0.7).add_(normal(rows, classes), alpha=1.5)
        t, ids = logits.topk(k, dim=1)
        # a teacher keeps as many classes as hold most of its probability; every sixteenth position it skips
        kept = torch.randint(1, k + 1, (rows, 1), generator=gen, device=DEVICE)
        kept[5::16] = 0
        s["teacher"] = t.contiguous()
        s["ids"] = torch.where(torch.arange(k, device=DEVICE) < kept, ids, -1).to(torch.int32)
        s["labels"] = torch.randint(0, classes, (rows,), generator=gen, device=DEVICE, dtype=torch.int32)
        return s
    width = (c["heads"] + 2 * c["kv_heads"]) * c["head"]
    s["x"] = normal(c["seqs"], c["tokens"] * width).to(_type(c))
    s["dy"] = normal(c["seqs"], c["tokens"] * c["heads"] * c["head"]).to(_type(c))
    if c["buckets"]:
        s["table"] = 0.5 * normal(c["heads"], c["buckets"])
        s["first"] = torch.tensor(_first_distances(c["buckets"], c["max_distance"]), device=DEVICE)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _attach_stage(s)
    return s


def _attach_stage(s):
    """The stage that a user's program keeps, with its input where the stage wants it."""
    from paper_2509_23241_amd.runner import GpuStage
    import numpy as np
    c = s["case"]
    common = dict(dtype=c["dtype"], n=1, stage_index=1, num_stages=2, policy="latest", lam=0.1, lr=0.0, momentum=0.0,
                  ring_capacity=1, max_in_flight=1, device=DEVICE)
    if c["kind"] == "distill":
        s["stage"] = st = GpuStage([(8, c["classes"], "none")],
                                   [np.zeros((c["classes"], 8), np.float32), np.zeros(c["classes"], np.float32)], mb=c["rows"], **common)
        st.forward(0, 0, torch.zeros(c["rows"], 8, dtype=st.tdtype, device=DEVICE))  # the loss belongs to a mini-batch in flight
        return
    layer = ("local", c["heads"] * c["head"], c["heads"], c["tokens"], c["kv_heads"], c["window"], c["sinks"], c["buckets"],
             c["max_distance"])
    params = [s["table"].cpu().numpy(), np.zeros(0, np.float32)] if c["buckets"] else []
    s["stage"] = st = GpuStage([layer], params, mb=c["seqs"], **common)
    view = st.input_view(0, 0)
    view.copy_(s["x"])
    s["x"], s["j"] = view, 0
    s["y"], s["dx"] = torch.empty_like(s["dy"]), torch.empty_like(view)


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _own_distill(state) if c["kind"] == "distill" else _own_attention(state)
    return _plain_distill(state) if c["kind"] == "distill" else _plain_attention(state)


def _own_attention(s):
    st, j = s["stage"], s["j"]
    s["j"] += 1
    st.forward(j, 0, s["x"], s["y"])
    st.backward(j, s["dy"], s["dx"])
    st.blend_update(j)
    out = {"y": s["y"], "dx": s["dx"]}
    if s["case"]["buckets"]:
        out["dtable"] = st.grad[: s["table"].numel()].view_as(s["table"])
    return out


def _own_distill(s):
    c = s["case"]
    loss, dlogits = s["stage"].loss_distill(0, s["logits"], s["teacher"], s["ids"], temperature=c["temperature"], labels=s["labels"],
                                            label_weight=c["label_weight"])
    return {"loss": loss, "dlogits": dlogits}


def _heads(x, c):
    """Queries, keys and values of all heads, [seqs, heads, tokens, head] in 32 bits."""
    h, kv, d = c["heads"], c["kv_heads"], c["head"]
    x = x.view(c["seqs"], c["tokens"], h + 2 * kv, d).transpose(1, 2).float()
    q, k, v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    return q, k.repeat_interleave(h // kv, 1), v.repeat_interleave(h // kv, 1)


def _plain_attention(s):
    c = s["case"]
    n, t, h, kv, d = c["seqs"], c["tokens"], c["heads"], c["kv_heads"], c["head"]
    scale = 1 / math.sqrt(d)
    q, k, v = _heads(s["x"], c)
    dy = s["dy"].view(n, t, h, d).transpose(1, 2).float().contiguous()
    at = torch.arange(t, device=DEVICE)
    distance = at[:, None] - at[None, :]
    hidden = distance < 0
    if c["window"]:
        hidden |= (distance >= c["window"]) & (at[None, :] >= c["sinks"])
    p = q @ k.transpose(2, 3).contiguous()
    p *= scale
    if c["buckets"]:
        bucket_at = (at[:, None] >= s["first"][None, 1:]).sum(1)
        p += s["table"][:, bucket_at][:, distance.clamp(min=0)]
    p.masked_fill_(hidden, -math.inf)
    p -= p.amax(3, keepdim=True)
    p.exp_()
    p /= p.sum(3, keepdim=True)
    y = p @ v
    ds = dy @ v.transpose(2, 3).contiguous()
    dv = p.transpose(2, 3).contiguous() @ dy
    ds -= (dy * y).sum(3, keepdim=True)
    ds *= p
    del p
    out = {"y": y.transpose(1, 2).reshape(n, -1).to(_type(c))}
    if c["buckets"]:
        # sums along the diagonals: row i shifted right by i, then columns
        total = ds.sum(0, dtype=torch.float64).flip(2)
        skewed = torch.nn.functional.pad(total, (0, t)).view(h, -1)[:, : t * (2 * t - 1)].view(h, t, 2 * t - 1)
        by_distance = skewed.sum(1)[:, t - 1:]
        one = (bucket_at[:, None] == torch.arange(c["buckets"], device=DEVICE)[None]).double()
        out["dtable"] = (by_distance @ one).float()
    ds *= scale
    dq = ds @ k
    dk = ds.transpose(2, 3).contiguous() @ q
    shared = (n, kv, h // kv, t, d)
    dx = torch.cat([dq, dk.view(shared).sum(2), dv.view(shared).sum(2)], 1)
    out["dx"] = dx.transpose(1, 2).reshape(n, -1).to(_type(c))
    return out


def _plain_distill(s):
    c = s["case"]
    rows, temperature, weight = c["rows"], c["temperature"], c["label_weight"]
    z = s["logits"].float()
    ids = s["ids"].long()
    stored = ids >= 0
    ids = ids.clamp(min=0)
    # the teacher's probabilities over the classes it kept; a row without any has no such term
    t = (s["teacher"] / temperature).masked_fill(~stored, -math.inf)
    has = stored.any(1, keepdim=True)
    e = torch.exp(t - t.amax(1, keepdim=True).masked_fill(~has, 0))
    p = e / e.sum(1, keepdim=True).masked_fill(~has, 1)
    top = z.amax(1, keepdim=True)
    soft = torch.exp((z - top) / temperature)
    total = soft.sum(1, keepdim=True)
    log_q = (z.gather(1, ids) - top) / temperature - total.log()
    kl = (torch.where(p > 0, p * (p.clamp(min=1e-38).log() - log_q), 0)).sum(1)
    grad = soft * (has / total * ((1 - weight) * temperature))
    grad.scatter_add_(1, ids, p * (-(1 - weight) * temperature))
    label = s["labels"].long()[:, None]
    hard = torch.exp(z - top)
    total = hard.sum(1, keepdim=True)
    ce = (total.log() - (z.gather(1, label) - top))[:, 0]
    grad += hard * (weight / total)
    grad.scatter_add_(1, label, torch.full_like(total, -weight))
    loss = (weight * ce.double() + (1 - weight) * temperature ** 2 * kl.double()).mean()
    return {"loss": loss.float().view(1), "dlogits": (grad / rows).to(_type(c))}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    c, s = case, _inputs(case, seed)
    return _exact_distill(c, s) if c["kind"] == "distill" else _exact_attention(c, s)


def _exact_attention(c, s):
    """Sequence by sequence and head by head, the gradients by differentiating the definition."""
    t, h, kv, d = c["tokens"], c["heads"], c["kv_heads"], c["head"]
    x = s["x"].double().view(c["seqs"], t, h + 2 * kv, d)
    dy = s["dy"].double().view(c["seqs"], t, h, d)
    y, dx = torch.empty_like(dy), torch.zeros_like(x)
    i = torch.arange(t, device=DEVICE).view(-1, 1)
    j = i.view(1, -1)
    visible = j <= i
    if c["window"]:
        visible = visible & ((j > i - c["window"]) | (j < c["sinks"]))
    bucket = torch.bucketize((i - j).clamp(min=0), s["first"], right=True) - 1 if c["buckets"] else None
    dtable = torch.zeros(h, c["buckets"], dtype=torch.float64, device=DEVICE)
    together = max(1, min(c["seqs"], 2 ** 26 // (t * t)))
    for a in range(0, c["seqs"], together):
        b = slice(a, min(a + together, c["seqs"]))
        for head in range(h):
            parts = [head, h + head // (h // kv), h + kv + head // (h // kv)]
            q, k, v = (x[b, :, at].clone().requires_grad_(True) for at in parts)
            score = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(d)
            leaves = [q, k, v]
            if c["buckets"]:
                shift = s["table"][head].double()[bucket].requires_grad_(True)
                score = score + shift
                leaves.append(shift)
            log_p = score.masked_fill(~visible, -math.inf).log_softmax(2)
            o = torch.matmul(log_p.exp(), v)
            grads = torch.autograd.grad(o, leaves, dy[b, :, head])
            y[b, :, head] = o.detach()
            for at, g in zip(parts, grads):
                dx[b, :, at] += g
            if c["buckets"]:
                for n in range(c["buckets"]):
                    dtable[head, n] += grads[3][bucket == n].sum()
            del score, log_p, o, grads, leaves
    out = {"y": y.view(c["seqs"], -1), "dx": dx.view(c["seqs"], -1)}
    if c["buckets"]:
        out["dtable"] = dtable
    return out


def _exact_distill(c, s):
    """Some rows at a time; the loss as defined, its gradient by differentiating it."""
    temperature, weight, rows = c["temperature"], c["label_weight"], c["rows"]
    dlogits = torch.empty(s["logits"].shape, dtype=torch.float64, device=DEVICE)
    loss = 0.0
    step = max(1, 2 ** 25 // c["classes"])
    for a in range(0, rows, step):
        b = slice(a, min(a + step, rows))
        z = s["logits"][b].double().requires_grad_(True)
        ids, teacher = s["ids"][b].long(), s["teacher"][b].double() / temperature
        kept = ids >= 0
        log_p = teacher.masked_fill(~kept, -1e300).log_softmax(1)
        p = log_p.exp() * kept
        log_q = (z / temperature).log_softmax(1).gather(1, ids.clamp(min=0))
        kl = (p * (log_p.masked_fill(~kept, 0) - log_q)).sum(1)
        ce = -z.log_softmax(1).gather(1, s["labels"][b].long()[:, None])[:, 0]
        part = (weight * ce + (1 - weight) * temperature ** 2 * kl).sum() / rows
        dlogits[b] = torch.autograd.grad(part, z)[0]
        loss += float(part.detach())
    return {"loss": torch.tensor([loss], dtype=torch.float64, device=DEVICE), "dlogits": dlogits}
