"""Timed cases of the operators between a mini-batch and a loss: attention to states of another length with a learned bias
by distance, that bias by itself, and the clipped policy loss of a model that chooses among candidates.

Attention. Batch entry b has `queries` tokens and `keys` states; `heads` query heads share `kv_heads` key/value heads
(heads / kv_heads query heads each). Only the states i < lengths[b] with mask[b][i] take part; a query without any gives
zeros. Bias: bucket(b, i, j) = how many of the ascending `bounds` are at most query_pos[b][i] - key_pos[b][j], and
table[head][bucket] is added to the scaled product.

Policy loss. Row r has a logit for each of its count[r] candidates (the rest is padding) and `picks` chosen ones (-1: none).
With l the log-softmax at the chosen candidate, ratio = exp(l - old), d = reference - l:
    loss = weight * (-min(ratio * advantage, clip(ratio, 1 - low, 1 + high) * advantage) + kl * (exp(d) - d - 1)).

Sizes are those of mini-batches as this package makes them (600 edges and up to 12 000 roots, 10 of 25 neighbors, hidden
width 100) and generic ones of token models.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04


def _attention(name, **more):
    case = dict(name=name, kind="attention", train=False, batch=1, queries=1, keys=1, heads=1, kv_heads=1, dim=64, dtype="bfloat16", buckets=0,
                positions="tokens", lengths="full", mask=False)
    case.update(more)
    return case


def _bias(name, **more):
    case = dict(name=name, kind="bias", train=False, batch=1, queries=1, keys=1, heads=1, dtype="bfloat16", buckets=32)
    case.update(more)
    return case


def _policy(name, **more):
    case = dict(name=name, kind="policy", rows=1, width=1, picks=1, dtype="bfloat16", ragged=False, reference=True)
    case.update(more)
    return case


def listed():
    return [
        # One query over a short encoded sequence: the smallest call of a service, where launches and host work count.
        _attention("answer_one", queries=1, keys=200, heads=8, kv_heads=8, dim=64, buckets=32),
        # A step of generation for 32 requests over encoded documents of other lengths, four query heads to a key head.
        _attention("answer_batch", batch=32, queries=1, keys=8192, heads=32, kv_heads=8, dim=128, lengths="ragged"),
        # Few requests over long documents in half precision: the work lies along the keys.
        _attention("answer_long", batch=2, queries=3, keys=100_001, heads=16, kv_heads=2, dim=128, dtype="float16", lengths="ragged", buckets=48),
        # The aggregation of a temporal graph model: each of a mini-batch's roots attends to its 10 sampled neighbors, 2 heads of 50,
        # biased by how long ago each interaction was; forward and backward in single precision.
        _attention("neighbors_train", train=True, batch=12_000, queries=1, keys=10, heads=2, kv_heads=2, dim=50, dtype="float32", buckets=16,
                   positions="times", lengths="counts"),
        # The same over candidate windows in half precision, one key head to two query heads; only the answer.
        _attention("candidates", batch=30_000, queries=1, keys=25, heads=4, kv_heads=2, dim=64, dtype="float16", buckets=24, positions="times",
                   lengths="counts"),
        # Encoder and decoder of middle length in single precision, odd sizes, padding inside the sequences.
        _attention("middle_train", train=True, batch=3, queries=333, keys=777, heads=6, kv_heads=3, dim=80, dtype="float32", lengths="ragged", mask=True),
        # A prompt over encoded documents, only the answer: matrix products bound it.
        _attention("prompt", batch=4, queries=2048, keys=4096, heads=16, kv_heads=16, dim=128, lengths="ragged"),
        # The largest: a training step over long sequences with bias, four query heads to a key head.
        _attention("long_train", train=True, batch=2, queries=4096, keys=4096, heads=16, kv_heads=4, dim=128, buckets=32),
        # The bias as a tensor, for a model that adds it itself, and the table's gradient from that tensor's.
        _bias("bias_tensor", queries=1024, keys=1024, heads=12),
        _bias("bias_gradient", train=True, batch=4, queries=1000, keys=2047, heads=16, dtype="float32"),
        # The policy of an adaptive sampler: 10 of 25 candidates chosen for each root.
        _policy("sampler_policy", rows=12_000, width=25, picks=10, dtype="float32", ragged=True, reference=False),
        # The policy of a token model: one chosen token a row, an odd vocabulary, a reference model.
        _policy("token_policy", rows=4096, width=64_001),
    ]


def _spread(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed()) / 2
    while True:
        shape = rng.choice(("answer", "neighbors", "train", "prompt", "bias", "policy_window", "policy_tokens"))
        dtype = rng.choice(("float32", "float16", "bfloat16", "bfloat16"))
        kv_heads = rng.choice((1, 2, 3, 4, 8))
        common = dict(dtype=dtype, kv_heads=kv_heads, heads=kv_heads * rng.choice((1, 1, 2, 4, 5)), dim=rng.choice((32, 50, 64, 64, 72, 96, 128, 128)),
                      buckets=rng.choice((0, 0, 2, 16, 32, 61)))
        if shape == "answer":
            case = _attention("", batch=_spread(rng, 1, 64), queries=rng.choice((1, 1, 1, 2, 5)), keys=_spread(rng, 1, 32_768), lengths=rng.choice(("full", "ragged")),
                              mask=rng.random() < 0.3, **common)
        elif shape == "neighbors":
            case = _attention("", train=rng.random() < 0.6, batch=_spread(rng, 600, 40_000), queries=1, keys=rng.randint(1, 64), lengths="counts", positions="times", **common)
        elif shape in ("train", "prompt"):
            case = _attention("", train=shape == "train", batch=rng.randint(1, 4), queries=_spread(rng, 1, 4096), keys=_spread(rng, 1, 4096),
                              lengths=rng.choice(("full", "ragged")), mask=rng.random() < 0.3, **common)
        elif shape == "bias":
            case = _bias("", train=rng.random() < 0.5, batch=rng.randint(1, 4), queries=_spread(rng, 1, 2048), keys=_spread(rng, 1, 2048), heads=rng.randint(1, 32), dtype=dtype,
                         buckets=rng.randint(2, 64))
        elif shape == "policy_window":
            width = rng.randint(2, 64)
            case = _policy("", rows=_spread(rng, 600, 100_000), width=width, picks=rng.randint(1, min(10, width)), dtype=dtype, ragged=True, reference=rng.random() < 0.5)
        else:
            case = _policy("", rows=_spread(rng, 1, 4096), width=_spread(rng, 100, 130_000), picks=rng.choice((1, 1, 4)), dtype=dtype, ragged=rng.random() < 0.3)
        del case["name"]
        if _cost(case) <= most and work(case)["bytes"] <= 2e9:
            return case


def _filled(case):
    """The share of the states that take part, on average."""
    share = {"full": 1.0, "ragged": 0.75, "counts": 0.8 + 0.15 * (case["keys"] + 1) / (2 * case["keys"])}[case["lengths"]]
    return share * (0.8 if case["mask"] else 1.0)


def work(case):
    if case["kind"] == "policy":
        r, w, n = case["rows"], case["width"], case["picks"]
        share = 0.75 if case["ragged"] else 1.0
        size = SIZE[case["dtype"]]
        return {"bytes": r * w * size * (1 + share) + r * n * (4 + 4 + 4 + 4 + 4 + 4 + (4 if case["reference"] else 0)), "flops": 8.0 * r * w * share}
    size, b, h, q, k = SIZE[case["dtype"]], case["batch"], case["heads"], case["queries"], case["keys"]
    if case["kind"] == "bias":
        return {"bytes": b * h * q * k * size + 8 * b * (q + k) + 2 * h * case["buckets"] * size, "flops": float(b * h * q * k)}
    d, seen = case["dim"], case["keys"] * _filled(case)
    rows = b * h * q * d * size
    states = b * case["kv_heads"] * d * size
    moved = 2 * rows + 2 * states * seen + (8 * b * (q + k) if case["buckets"] else 0) + (b * k if case["mask"] else 0)
    if case["train"]:   # forward and backward both read their inputs; the gradients are written whole
        moved += 4 * rows + 2 * states * seen + 2 * states * k
    return {"bytes": moved, "flops": (14.0 if case["train"] else 4.0) * b * h * q * seen * d}


def _positions(case, g, lengths):
    b, q, k = case["batch"], case["queries"], case["keys"]
    if case.get("positions") == "times":   # query times in seconds over some years; neighbors' before them, the latest first
        now = torch.randint(200_000_000, 1_000_000_000, (b, q), generator=g, device="cuda")
        back = torch.exp(torch.rand((b, k), generator=g, device="cuda", dtype=torch.float64) * 17).long()
        return now, now[:, :1] - 1 - torch.sort(back, dim=1).values
    if q <= 5:   # the query follows the states
        start = torch.randint(0, 1000, (b, 1), generator=g, device="cuda") + k
        return start + torch.arange(q, device="cuda"), torch.arange(k, device="cuda").expand(b, k).contiguous()
    shift = torch.randint(0, 1000, (1, 1), generator=g, device="cuda")   # shared by the batch
    return shift + torch.arange(q, device="cuda")[None], shift + torch.arange(k, device="cuda")[None]


def _bounds(case):
    """Ascending bounds: small distances apart, larger ones by the logarithm, to both sides where tokens are compared."""
    n = case["buckets"] - 1
    if case.get("positions") == "times":
        steps = [round(math.exp((i + 1) * 17 / (n + 1))) for i in range(n)]
    else:
        near, far = n // 2, n - n // 2
        steps = [-round(1.3 ** i + i) for i in range(near)][::-1] + [round(1.3 ** i + i) for i in range(far)]
    for i in range(1, n):
        steps[i] = max(steps[i], steps[i - 1] + 1)
    return torch.tensor(steps, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)

    s = dict(case)
    if case["kind"] == "policy":
        r, w, n = case["rows"], case["width"], case["picks"]
        s["logits"] = normal(r, w, scale=2.0)
        s["count"] = torch.randint(w // 2, w + 1, (r,), generator=g, device="cuda", dtype=torch.int32) if case["ragged"] else None
        width = s["count"].long() if case["ragged"] else torch.full((r,), w, device="cuda")
        picks = (torch.rand((r, n), generator=g, device="cuda") * width[:, None]).long()
        picks = torch.minimum(picks, (width - 1).clamp(min=0)[:, None])
        free = torch.arange(n, device="cuda")[None] >= width[:, None]
        if n > 1:   # a row's choices are neighboring candidates, each once; fewer where there are fewer candidates
            first = (picks[:, :1]).clamp(max=0) + (torch.rand((r, 1), generator=g, device="cuda") * (width - n + 1).clamp(min=1)[:, None]).long()
            picks = first + torch.arange(n, device="cuda")[None]
        s["actions"] = torch.where(free, -1, picks).int()
        inside = torch.arange(w, device="cuda")[None] < width[:, None]
        chosen = torch.empty((r, n), device="cuda")
        for i in range(0, r, 512):   # the log-probabilities of a model some steps older: near the present ones
            x = torch.where(inside[i:i + 512], s["logits"][i:i + 512].float(), -math.inf)
            chosen[i:i + 512] = torch.gather(torch.log_softmax(x, 1), 1, picks[i:i + 512].clamp(0, w - 1))
        chosen = torch.where(free, 0.0, chosen)
        s["old"] = chosen + normal(r, n, scale=0.2, dtype=torch.float32)
        s["ref"] = chosen + normal(r, n, scale=0.3, dtype=torch.float32) if case["reference"] else None
        s["advantage"] = normal(r, n, dtype=torch.float32)
        s["weight"] = torch.full((r, n), 1.0 / (r * n), device="cuda") * (torch.rand((r, n), generator=g, device="cuda") < 0.9)
        return s
    b, q, k, h = case["batch"], case["queries"], case["keys"], case["heads"]
    lengths = None
    if case["kind"] == "attention":
        kv, d = case["kv_heads"], case["dim"]
        s["q"] = normal(b, q, h, d)
        both = normal(b, k, 2, kv, d)   # keys and values side by side, as one projection leaves them
        s["k"], s["v"] = both[:, :, 0], both[:, :, 1]
        if case["lengths"] == "ragged":
            lengths = torch.randint((k + 1) // 2, k + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        elif case["lengths"] == "counts":   # most roots have as many neighbors as are asked for, some fewer, some none
            part = torch.randint(1, k + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
            u = torch.rand((b,), generator=g, device="cuda")
            lengths = torch.where(u < 0.05, 0, torch.where(u < 0.2, part, k)).int()
        s["lengths"] = lengths
        s["mask"] = torch.rand((b, k), generator=g, device="cuda") < 0.8 if case["mask"] else None
        if case["train"]:
            s["dout"] = normal(b, q, h, d)
    if case["buckets"]:
        s["query_pos"], s["key_pos"] = _positions(case, g, lengths)
        s["bounds"] = _bounds(case)
        s["table"] = normal(h, case["buckets"])
    if case["kind"] == "bias":
        if b > 1:   # a position of its own for each entry
            s["query_pos"] = s["query_pos"] + torch.randint(0, 50, (b, 1), generator=g, device="cuda")
            s["key_pos"] = s["key_pos"].expand(b, k).contiguous()
        if case["train"]:
            s["dbias"] = normal(b, h, q, k)
    return s


# ---- the plain forms -----------------------------------------------------------------------

def _buckets(s):
    apart = s["query_pos"][:, :, None] - s["key_pos"][:, None, :]
    return torch.bucketize(apart, s["bounds"], right=True)   # [B or 1, queries, keys]


def _plain_bias(s, bucket):
    return s["table"].float()[:, bucket].transpose(0, 1)      # [B or 1, heads, queries, keys]


def _plain_bias_gradient(s, bucket, dbias):
    """dbias float32[B, heads, queries, keys] -> [heads, buckets], as a product with the buckets' indicator."""
    rows = dbias.permute(0, 2, 1, 3).contiguous()                                     # [B, queries, heads, keys]
    which = (bucket[..., None] == torch.arange(s["buckets"], device="cuda")).float()   # [B or 1, queries, keys, buckets]
    return torch.matmul(rows, which).sum((0, 1)).to(s["table"].dtype)


def _plain_attention(s):
    b, q, k, h, kv, d = (s[x] for x in ("batch", "queries", "keys", "heads", "kv_heads", "dim"))
    g, scale = h // kv, 1 / math.sqrt(d)

    def by_head(x):   # [B, queries, heads, d] -> [B, kv_heads, queries * g, d]
        return x.float().view(b, q, kv, g, d).permute(0, 2, 1, 3, 4).reshape(b, kv, q * g, d)

    def back(x):
        return x.view(b, kv, q, g, d).permute(0, 2, 1, 3, 4).reshape(b, q, h, d)

    seen = torch.ones((b, k), dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        seen = torch.arange(k, device="cuda")[None] < s["lengths"][:, None]
    if s["mask"] is not None:
        seen = seen & s["mask"]
    keys = torch.where(seen[:, :, None, None], s["k"].float(), 0.0).transpose(1, 2).contiguous()      # [B, kv_heads, keys, d]
    values = torch.where(seen[:, :, None, None], s["v"].float(), 0.0).transpose(1, 2).contiguous()
    queries = by_head(s["q"])
    x = torch.matmul(queries, keys.transpose(2, 3)) * scale
    if s["buckets"]:
        bucket = _buckets(s)
        bias = _plain_bias(s, bucket)                                                               # [B or 1, heads, queries, keys]
        x = x + bias.unflatten(1, (kv, g)).transpose(2, 3).reshape(-1, kv, q * g, k)
    x = torch.where(seen[:, None, None, :], x, -math.inf)
    top = x.amax(3, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p, values)
    got = {"out": back(o).to(s["q"].dtype)}
    if s["train"]:
        do = by_head(s["dout"])
        dp = torch.matmul(do, values.transpose(2, 3))
        dx = p * (dp - (do * o).sum(3, keepdim=True))
        got["dq"] = back(torch.matmul(dx, keys) * scale).to(s["q"].dtype)
        got["dk"] = (torch.matmul(dx.transpose(2, 3), queries) * scale).transpose(1, 2).to(s["q"].dtype)
        got["dv"] = torch.matmul(p.transpose(2, 3), do).transpose(1, 2).to(s["q"].dtype)
        if s["buckets"]:
            got["dtable"] = _plain_bias_gradient(s, bucket, dx.view(b, kv, q, g, k).permute(0, 1, 3, 2, 4).reshape(b, h, q, k))
    return got


def _plain_policy(s):
    w = s["width"]
    x = s["logits"].float()
    if s["count"] is not None:
        x = torch.where(torch.arange(w, device="cuda")[None] < s["count"][:, None], x, -math.inf)
    top = x.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    none, at = s["actions"] < 0, s["actions"].clamp(min=0).long()
    logp = torch.gather(x, 1, at) - top - torch.log(total)
    ratio = torch.exp(logp - s["old"])
    a = s["advantage"]
    whole, cut = ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    loss, slope = -torch.minimum(whole, cut), torch.where(whole <= cut, -whole, 0.0)
    if s["ref"] is not None:
        apart = s["ref"] - logp
        loss, slope = loss + KL * (torch.exp(apart) - apart - 1), slope + KL * (1 - torch.exp(apart))
    loss, slope, logp = (torch.where(none, 0.0, y) for y in (loss * s["weight"], slope * s["weight"], logp))
    grad = e / torch.where(total == 0, 1.0, total) * -slope.sum(1, keepdim=True)
    grad = grad.scatter_add(1, at, slope)
    return {"loss": loss, "logp": logp, "grad": grad.to(s["logits"].dtype)}


# ---- one pass --------------------------------------------------------------------------------

def run(state):
    s = state
    if not own:
        if s["kind"] == "policy":
            return _plain_policy(s)
        if s["kind"] == "attention":
            return _plain_attention(s)
        if s["train"]:
            return {"dtable": _plain_bias_gradient(s, _buckets(s), s["dbias"].float())}
        return {"bias": _plain_bias(s, _buckets(s)).to(s["table"].dtype)}
    import paper_2402_05396_amd as T
    if s["kind"] == "policy":
        loss, logp, grad = T.policy_loss(s["logits"], s["actions"], s["advantage"], s["old"], s["ref"], count=s["count"], weight=s["weight"], clip_low=CLIP_LOW,
                                         clip_high=CLIP_HIGH, kl=KL if s["reference"] else 0.0)
        return {"loss": loss, "logp": logp, "grad": grad}
    if s["kind"] == "bias":
        if s["train"]:
            return {"dtable": T.relative_bias_grad(s["dbias"], s["bounds"], s["query_pos"], s["key_pos"])}
        return {"bias": T.relative_bias(s["table"], s["bounds"], s["query_pos"], s["key_pos"])}
    bias = (s["table"], s["bounds"], s["query_pos"], s["key_pos"]) if s["buckets"] else None
    if not s["train"]:
        return {"out": T.cross_attention(s["q"], s["k"], s["v"], lengths=s["lengths"], mask=s["mask"], bias=bias)}
    out, stats = T.cross_attention(s["q"], s["k"], s["v"], lengths=s["lengths"], mask=s["mask"], bias=bias, want_stats=True)
    dq, dk, dv, dtable = T.cross_attention_grad(s["dout"], s["q"], s["k"], s["v"], out, stats, lengths=s["lengths"], mask=s["mask"], bias=bias)
    got = {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if bias:
        got["dtable"] = dtable
    return got


# ---- the definition, in 64 bits ----------------------------------------------------------------

def _exact_distance_bias(s, b):
    """float64 [heads, queries, keys] of batch entry b and the bucket of each pair, counted bound by bound."""
    apart = s["query_pos"][b % len(s["query_pos"])][:, None] - s["key_pos"][b % len(s["key_pos"])][None, :]
    bucket = torch.zeros_like(apart)
    for bound in s["bounds"].tolist():
        bucket += (apart >= bound).long()
    return s["table"].double()[:, bucket], bucket


def _exact_by_bucket(buckets, bucket, grad):
    return torch.stack([(grad * (bucket == i)).sum(dim=tuple(range(1, grad.dim()))) for i in range(buckets)], 1)


def _exact_attention_many(s):
    """Many short rows, one query each: all at once."""
    h, g = s["heads"], s["heads"] // s["kv_heads"]
    leaf = {n: s[n].double().requires_grad_(s["train"]) for n in ("q", "k", "v")}
    keys, values = (leaf[n].repeat_interleave(g, 2) for n in ("k", "v"))
    x = (leaf["q"] * keys).sum(3) / s["dim"] ** 0.5                  # [B, keys, heads]
    if s["buckets"]:
        apart = s["query_pos"] - s["key_pos"]
        bucket = sum((apart >= bound).long() for bound in s["bounds"].tolist())
        bias = s["table"].double().t()[bucket].requires_grad_(s["train"])
        x = x + bias
    seen = torch.arange(s["keys"], device="cuda")[None] < s["lengths"][:, None].long()
    x = x.masked_fill(~seen[:, :, None], -1e300)
    p = torch.softmax(x, 1) * seen[:, :, None]
    out = (p[..., None] * values).sum(1, keepdim=True)
    got = {"out": out.detach()}
    if s["train"]:
        wanted = [leaf["q"], leaf["k"], leaf["v"]] + ([bias] if s["buckets"] else [])
        grads = torch.autograd.grad(out, wanted, s["dout"].double())
        got.update(zip(("dq", "dk", "dv"), grads))
        if s["buckets"]:
            got["dtable"] = _exact_by_bucket(s["buckets"], bucket[None], grads[3].permute(2, 0, 1).contiguous())
    return got


def _exact_attention(s):
    if s["lengths"] is not None and s["batch"] >= 600 and s["queries"] == 1:
        return _exact_attention_many(s)
    b, h, g = s["batch"], s["heads"], s["heads"] // s["kv_heads"]
    parts = {n: [] for n in ("out", "dq", "dk", "dv")}
    dtable = 0
    for i in range(b):
        n = s["keys"] if s["lengths"] is None else int(s["lengths"][i])
        at = torch.arange(n, device="cuda")
        if s["mask"] is not None:
            at = at[s["mask"][i, :n]]
        q = s["q"][i].double().transpose(0, 1).contiguous().requires_grad_(s["train"])                            # [heads, queries, d]
        k, v = (s[x][i][at].double().transpose(0, 1).contiguous().requires_grad_(s["train"]) for x in ("k", "v"))   # [kv_heads, seen, d]
        out = []
        if s["buckets"]:
            bias, bucket = _exact_distance_bias(s, i)
            bias, bucket = bias[:, :, at].requires_grad_(s["train"]), bucket[:, at]
        for j in range(h):
            x = q[j] @ k[j // g].t() * s["dim"] ** -0.5
            if s["buckets"]:
                x = x + bias[j]
            out.append(torch.softmax(x, 1) @ v[j // g] if len(at) else torch.zeros_like(q[j]) + q[j] * 0)
        out = torch.stack(out)
        parts["out"].append(out.detach().transpose(0, 1))
        if s["train"]:
            wanted = [q, k, v] + ([bias] if s["buckets"] else [])
            grads = torch.autograd.grad(out, wanted, s["dout"][i].double().transpose(0, 1).contiguous(), allow_unused=True, materialize_grads=True)
            parts["dq"].append(grads[0].transpose(0, 1))
            for name, grad in zip(("dk", "dv"), grads[1:3]):
                whole = torch.zeros((s["keys"], s["kv_heads"], s["dim"]), dtype=torch.float64, device="cuda")
                whole[at] = grad.transpose(0, 1)
                parts[name].append(whole)
            if s["buckets"]:
                dtable = dtable + _exact_by_bucket(s["buckets"], bucket[None], grads[3])
    got = {n: torch.stack(x) for n, x in parts.items() if x}
    if s["train"] and s["buckets"]:
        got["dtable"] = dtable
    return got


def _exact_policy(s):
    losses, logps, grads = [], [], []
    for i in range(0, s["rows"], 256):
        x = s["logits"][i:i + 256].double().requires_grad_()
        kept = x
        if s["count"] is not None:
            kept = x.masked_fill(torch.arange(s["width"], device="cuda") >= s["count"][i:i + 256, None], -1e300)
        chosen = s["actions"][i:i + 256].long()
        given = chosen >= 0
        logp = torch.log_softmax(kept, 1).gather(1, chosen.clamp(min=0))
        gain = s["advantage"][i:i + 256].double()
        ratio = (logp - s["old"][i:i + 256].double()).exp()
        best = torch.where(gain >= 0, ratio.clamp(max=1 + CLIP_HIGH), ratio.clamp(min=1 - CLIP_LOW)) * gain
        loss = -best
        if s["ref"] is not None:
            apart = s["ref"][i:i + 256].double() - logp
            loss = loss + KL * (apart.exp() - 1 - apart)
        loss = torch.where(given, loss * s["weight"][i:i + 256].double(), 0.0)
        grads.append(torch.autograd.grad(loss.sum(), x)[0])
        losses.append(loss.detach())
        logps.append(torch.where(given, logp, 0.0).detach())
    return {"loss": torch.cat(losses), "logp": torch.cat(logps), "grad": torch.cat(grads)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "policy":
        return _exact_policy(s)
    if case["kind"] == "attention":
        return _exact_attention(s)
    found = [_exact_distance_bias(s, i) for i in range(max(len(s["query_pos"]), len(s["key_pos"])))]
    if not case["train"]:
        return {"bias": torch.stack([x for x, _ in found])}
    return {"dtable": sum(_exact_by_bucket(case["buckets"], bucket[None], s["dbias"][i].double()) for i, (_, bucket) in enumerate(found))}
