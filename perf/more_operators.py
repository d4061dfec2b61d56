"""Timed cases of the operators around a model's step: layer norm with its gradient, draws of a policy's actions with temperature,
top-k, top-p and min-p, and the AdamW step over a list of tensors with moments in 32 or in 8 bits.

Layer norm, a row x of `width` elements:
    mean = sum(x) / width, rstd = (sum((x - mean)^2) / width + eps)^-1/2, xhat = (x - mean) rstd, out = xhat weight + bias
    with g = dout weight: dx = rstd (g - mean(g) - xhat mean(g xhat)), dweight = sum over rows of dout xhat, dbias = sum over rows of dout.

Draws. Row r has logits x[c] for its count[r] candidates. In order of falling x (ties: the lower index first), w = exp((x - max x) / temperature):
top-k keeps the first k; top-p of these the first ones, as few as hold a share p of their sum; min-p of these the ones with w >= min_p. The
action for the number u in [0, 1) is the first kept candidate by index whose running sum of w exceeds u times the whole sum. A temperature
of 0 takes the largest. With it comes the log-probability in the softmax of the row as it is: what a clipped policy loss is given later.

AdamW at step t, with g the gradient times a factor:
    m = beta1 m + (1 - beta1) g, v = beta2 v + (1 - beta2) g^2
    p = p (1 - lr weight_decay) - (lr / (1 - beta1^t)) m / (sqrt(v / (1 - beta2^t)) + eps)
Moments in 8 bits: 256 neighbors share a unit for each moment. m = sign c^2 unit (c < 128, bit 7 the sign), sqrt(v) = c^2 unit (c < 256), the unit such
that the largest has the largest c. After the step a moment goes to one of its two neighboring codes, by chance, so that its expectation is
the moment: the chance is 16 bits of Philox 4x32-10, key seed, counter (element / 8, tensor's number, step, tag), bits 16 (element % 8).

Sizes are those of this package's mini-batches (12 000 roots, 25 candidates, hidden width 100) and generic ones of token models.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}
EPS = 1e-5
BETA1, BETA2, ADAM_EPS, DECAY, LR = 0.9, 0.999, 1e-8, 0.01, 1e-4
BLOCK, TAG = 256, 0x4144414D


def _norm(name, **more):
    case = dict(name=name, kind="norm", train=False, rows=1, width=1, pad=0, dtype="bfloat16", weights="same")
    case.update(more)
    return case


def _draws(name, **more):
    case = dict(name=name, kind="draws", rows=1, width=1, picks=1, dtype="bfloat16", ragged=False, mixed=False, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    case.update(more)
    return case


def _adamw(name, **more):
    case = dict(name=name, kind="adamw", layers=1, width=100, dtype="float32", grads="same", bits=32)
    case.update(more)
    return case


def listed():
    return [
        # One token's hidden state: the smallest call of a service.
        _norm("norm_one", width=4096),
        # The states of 12 000 roots of a temporal graph model, forward and backward in single precision.
        _norm("norm_roots_train", train=True, rows=12_000, width=100, dtype="float32"),
        # Odd sizes in half precision, rows inside a wider projection.
        _norm("norm_odd_train", train=True, rows=3001, width=1023, pad=9, dtype="float16"),
        # A prompt's tokens, only the answer.
        _norm("norm_prompt", rows=8192, width=5120),
        # Tokens of a training step, weights kept in single precision.
        _norm("norm_tokens_train", train=True, rows=16_384, width=4096, weights="float32"),
        # The adaptive sampler's choice: 10 draws among up to 25 candidates of each root.
        _draws("draw_candidates", rows=12_000, width=25, picks=10, dtype="float32", ragged=True, temperature=0.8, top_p=0.95),
        # The next token of one request: latency.
        _draws("draw_token", width=64_001, temperature=0.7, top_k=50, top_p=0.9),
        # The next tokens of 64 requests, each with settings of its own.
        _draws("draw_requests", rows=64, width=130_000, dtype="float32", mixed=True),
        # Tokens for a policy's training: one draw from each of many rows, the tail cut off.
        _draws("draw_rollout", rows=4096, width=64_001, top_p=0.95),
        # The parameters of a temporal graph model, many small tensors.
        _adamw("adamw_graph", layers=4, width=100),
        # Layers of a token model: matrices in bfloat16, the rest in single precision, moments in 32 bits.
        _adamw("adamw_layers", layers=8, width=1024, dtype="bfloat16"),
        # Parameters in single precision with gradients in bfloat16, moments in 8 bits (which are returned as what they stand for).
        _adamw("adamw_bytes", layers=6, width=1280, grads="bfloat16", bits=8),
    ]


def _spread(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _cost(case):
    return work(case)["bytes"]


def draw(rng):
    while True:
        shape = rng.choice(("norm_short", "norm_long", "norm_long", "draws_window", "draws_tokens", "draws_tokens", "adamw"))
        dtype = rng.choice(("float32", "float16", "bfloat16", "bfloat16"))
        if shape == "norm_short":
            case = _norm("", train=rng.random() < 0.6, rows=_spread(rng, 600, 200_000), width=rng.randint(1, 256), pad=rng.choice((0, 0, 3)), dtype=dtype,
                         weights=rng.choice(("same", "float32")))
        elif shape == "norm_long":
            case = _norm("", train=rng.random() < 0.6, rows=_spread(rng, 1, 16_384), width=_spread(rng, 256, 20_000), pad=rng.choice((0, 0, 8, 5)), dtype=dtype,
                         weights=rng.choice(("same", "float32")))
        elif shape == "draws_window":
            case = _draws("", rows=_spread(rng, 600, 100_000), width=rng.randint(2, 64), picks=rng.randint(1, 10), dtype=dtype, ragged=True)
        elif shape == "draws_tokens":
            case = _draws("", rows=_spread(rng, 1, 4096), width=_spread(rng, 65, 130_000), picks=rng.choice((1, 1, 4)), dtype=dtype, ragged=rng.random() < 0.2, mixed=rng.random() < 0.4)
        else:
            case = _adamw("", layers=rng.randint(1, 8), width=_spread(rng, 20, 1300), dtype=dtype, bits=rng.choice((8, 32)))
            if dtype == "float32":
                case["grads"] = rng.choice(("same", "bfloat16", "float16"))
        if case["kind"] == "draws" and not case["mixed"]:
            case.update(temperature=rng.choice((0.0, 0.3, 0.7, 1.0, 1.0, 1.4)), top_k=rng.choice((0, 0, 1, 5, 50, 300)), top_p=rng.choice((1.0, 1.0, 0.5, 0.9, 0.95)),
                        min_p=rng.choice((0.0, 0.0, 0.02, 0.1)))
        del case["name"]
        if _cost(case) <= most_of(case["kind"]):
            return case


def most_of(kind):
    """What the largest listed case of a kind moves."""
    return max(_cost(c) for c in listed() if c["kind"] == kind)


def _sizes(case):
    """The elements of each tensor of a model: (matrices, vectors)."""
    w = case["width"]
    matrices = [w * w, w * w, w * w, w * w, 4 * w * w, 4 * w * w] * case["layers"]
    return matrices, [w, w, 4 * w, w, w, w] * case["layers"]


def work(case):
    if case["kind"] == "norm":
        size = SIZE[case["dtype"]]
        n, weight = case["rows"] * case["width"], 2 * case["width"] * (size if case["weights"] == "same" else 4)
        if not case["train"]:
            return {"bytes": 2 * n * size + weight, "flops": 8.0 * n}
        return {"bytes": 5 * n * size + 3 * weight + 16 * case["rows"], "flops": 22.0 * n}
    if case["kind"] == "draws":
        n = case["rows"] * case["width"] * (0.75 if case["ragged"] else 1.0)
        return {"bytes": n * SIZE[case["dtype"]] + case["rows"] * case["picks"] * 12, "flops": 12.0 * n}
    matrices, vectors = (sum(x) for x in _sizes(case))
    size, moved = SIZE[case["dtype"]], 0
    grad = size if case["grads"] == "same" else SIZE[case["grads"]]
    moment = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 2 + 8 / BLOCK + 4   # 8 bits: read, written, and read again and returned in 16
    for n, p, g in ((matrices, size, grad), (vectors, 4, grad if case["dtype"] == "float32" else 4)):
        moved += n * (2 * p + g + moment)
    return {"bytes": moved, "flops": 14.0 * (matrices + vectors)}


# ---- what a user's program has in hand ---------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = dict(case)
    if case["kind"] == "norm":
        r, w = case["rows"], case["width"]
        wide = normal(r, w + case["pad"])
        wide *= 0.5 + uniform(r, 1) * 2   # rows of other sizes, some elements always large, none around zero
        wide += 0.3 + 4 * (uniform(1, w + case["pad"]) < 0.01)
        s["x"] = wide.to(dt)[:, case["pad"]:]
        kept = dt if case["weights"] == "same" else torch.float32
        s["weight"], s["bias"] = (1 + 0.2 * normal(w)).to(kept), normal(w, scale=0.2).to(kept)
        if case["train"]:
            s["dout"] = normal(r, w, dtype=dt)
    elif case["kind"] == "draws":
        r, w = case["rows"], case["width"]
        s["logits"] = (normal(r, w) * (1 + 2 * uniform(r, 1))).to(dt)   # some rows flat, some with few likely candidates
        s["count"] = None
        if case["ragged"]:   # most rows are full, some have fewer candidates, some none
            part = torch.randint(1, w + 1, (r,), generator=g, device="cuda")
            share = uniform(r)
            s["count"] = torch.where(share < 0.02, 0, torch.where(share < 0.5, part, w)).int()
        s["uniform"] = uniform(r, case["picks"])
        if case["mixed"]:
            def some(share, values, other):
                return torch.where(uniform(r) < share, values, other)
            s["temperature"] = some(0.9, 0.3 + uniform(r), torch.zeros((), device="cuda"))
            s["top_k"] = some(0.5, torch.randint(1, 200, (r,), generator=g, device="cuda", dtype=torch.int32), torch.zeros((), device="cuda", dtype=torch.int32))
            s["top_p"] = some(0.6, 0.5 + 0.49 * uniform(r), torch.ones((), device="cuda"))
            s["min_p"] = some(0.4, 0.1 * uniform(r), torch.zeros((), device="cuda"))
    else:
        s["step"] = 1000 + seed % 1000
        s["groups"] = []
        s["params"], s["grads"], s["m"], s["v"], s["units"] = [], [], [], [], ([], [])
        first = 0
        for sizes, p_type in zip(_sizes(case), (dt, torch.float32)):
            g_type = p_type if case["grads"] == "same" or case["dtype"] != "float32" else DTYPES[case["grads"]]
            # All tensors of a type in one buffer, each from a whole block on.
            blocks = [-(-n // BLOCK) for n in sizes]
            total = sum(blocks)
            number = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor(blocks, device="cuda"))
            start = torch.tensor(blocks, device="cuda").cumsum(0) - torch.tensor(blocks, device="cuda")
            place = torch.arange(total, device="cuda") - start[number]
            inside = place[:, None] * BLOCK + torch.arange(BLOCK, device="cuda") < torch.tensor(sizes, device="cuda")[number][:, None]
            grow = torch.exp(normal(total, 1) - 7)   # gradients of other sizes in other places
            grad = normal(total, BLOCK) * grow * inside
            q = {"number": number + first, "place": place, "p": (normal(total, BLOCK, scale=0.05) * inside).to(p_type), "g": grad.to(g_type)}
            if case["bits"] == 32:
                q["m"] = normal(total, BLOCK) * 0.3 * grow * inside
                q["v"] = ((0.5 + uniform(total, BLOCK)) * grow) ** 2 * inside
            else:
                cv = torch.randint(60, 256, (total, BLOCK), generator=g, device="cuda")
                cm = (cv * uniform(total, BLOCK) * (127 / 255)).long()
                q["v"] = (cv * inside).to(torch.uint8)
                q["m"] = ((cm + 128 * (uniform(total, BLOCK) < 0.5)) * inside).to(torch.uint8)
                q["v_unit"], q["m_unit"] = 2 * grow[:, 0] / 255 ** 2, 0.8 * grow[:, 0] / 127 ** 2
            s["groups"].append(q)
            at = 0
            for n, b in zip(sizes, blocks):
                for name, to in (("p", "params"), ("g", "grads"), ("m", "m"), ("v", "v")):
                    s[to].append(q[name].view(-1)[at * BLOCK:at * BLOCK + n])
                if case["bits"] == 8:
                    s["units"][0].append(q["m_unit"][at:at + b])
                    s["units"][1].append(q["v_unit"][at:at + b])
                at += b
            first += len(sizes)
    return s


# ---- the plain forms -----------------------------------------------------------------------

def _plain_norm(s):
    x, weight = s["x"].float(), s["weight"].float()
    mean = x.sum(1, keepdim=True) / s["width"]
    away = x - mean
    rstd = 1 / torch.sqrt((away * away).sum(1, keepdim=True) / s["width"] + EPS)
    xhat = away * rstd
    got = {"out": (xhat * weight + s["bias"].float()).to(s["x"].dtype)}
    if s["train"]:
        dout = s["dout"].float()
        g = dout * weight
        part = (g * xhat).sum(1, keepdim=True) / s["width"]
        got["dx"] = (rstd * (g - g.sum(1, keepdim=True) / s["width"] - xhat * part)).to(s["x"].dtype)
        got["dweight"] = (dout * xhat).sum(0).to(s["weight"].dtype)
        got["dbias"] = dout.sum(0).to(s["weight"].dtype)
    return got


def _settings(s):
    """temperature, top_k, top_p, min_p as a column each, in 64 bits."""
    if s["mixed"]:
        return [s[n].double()[:, None] for n in ("temperature", "top_k", "top_p", "min_p")]
    column = torch.ones((s["rows"], 1), dtype=torch.float32, device="cuda")
    return [(column * s[n]).double() for n in ("temperature", "top_k", "top_p", "min_p")]


def _plain_draws(s):
    w = s["width"]
    temperature, top_k, top_p, min_p = _settings(s)
    x = s["logits"].float()
    if s["count"] is not None:
        x = torch.where(torch.arange(w, device="cuda") < s["count"][:, None], x, -math.inf)
    top = x.amax(1, keepdim=True)
    none = top == -math.inf
    top = torch.where(none, 0.0, top).double()
    falling, at = torch.sort(x, dim=1, descending=True, stable=True)
    rank = torch.arange(w, device="cuda")
    chance = torch.exp((falling.double() - top) / torch.where(temperature > 0, temperature, 1.0))
    chance = torch.where((temperature > 0) | (rank == 0), chance, 0.0)
    kept = torch.where((rank < top_k) | (top_k == 0), chance, 0.0)
    upto = kept.cumsum(1)
    before = torch.cat([torch.zeros_like(top), upto[:, :-1]], 1)
    keep = (top_p >= 1) | (before < top_p * upto[:, -1:]) | (rank == 0)
    keep = keep & ((chance >= min_p) | (rank == 0))
    kept = torch.where(keep, kept, 0.0)
    running = torch.zeros_like(kept).scatter(1, at, kept).cumsum(1)
    whole = running[:, -1:]
    action = torch.searchsorted(running, s["uniform"].double() * whole, right=True)
    action = torch.minimum(action, (running < whole).sum(1, keepdim=True))   # no further than the last one kept
    none = none.expand_as(action)
    action = torch.where(none, 0, action)
    apart = x.double() - top
    logp = torch.gather(apart, 1, action) - torch.log(torch.exp(apart).sum(1, keepdim=True))
    return {"action": torch.where(none, -1, action).int(), "logp": torch.where(none, 0.0, logp).float()}


def _plain_philox(piece, number, step, seed):
    """Four words of 32 bits for each counter (piece, number, step, TAG), as 64-bit integers."""
    low = 0xFFFFFFFF
    c = [piece & low, number & low, torch.full_like(piece, step & low), torch.full_like(piece, TAG)]
    keys = [seed & low, seed >> 32 & low]
    for i in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57   # 64 bits of each product, also where the sign bit is one of them
        c = [(b >> 32 & low) ^ c[1] ^ keys[0], b & low, (a >> 32 & low) ^ c[3] ^ keys[1], a & low]
        keys = [(keys[0] + 0x9E3779B9) & low, (keys[1] + 0xBB67AE85) & low]
    return c


def _plain_chance(q, step):
    """[blocks, 256] numbers in (0, 1), 16 bits of a draw each."""
    piece = q["place"][:, None] * (BLOCK // 8) + torch.arange(BLOCK // 8, device="cuda")
    words = torch.stack(_plain_philox(piece, q["number"][:, None].expand_as(piece), step, 0), 2)      # [blocks, 32, 4]
    halves = torch.stack([words & 0xFFFF, words >> 16], 3).reshape(-1, BLOCK)
    return (halves.float() + 0.5) * (1 / 65536)


def _plain_code(root, most, unit, chance, power):
    """Codes for numbers root = unit c^2 (c in 0 .. most, between two codes by chance, so that root^power has its expectation)."""
    y = root * torch.where(unit > 0, 1 / unit, 0.0)[:, None]
    c = torch.floor(torch.sqrt(y)).clamp(max=most - 1)
    low, high = c * c, (c + 1) * (c + 1)
    if power == 2:
        y, low, high = y * y, low * low, high * high
    return torch.where(y - low > chance * (high - low), c + 1, c)


def _plain_adamw(s):
    step = s["step"]
    got, b1, b2 = {}, 1 - BETA1 ** step, 1 - BETA2 ** step
    for i, q in enumerate(s["groups"]):
        p, g, m, v = (q[n].float() for n in ("p", "g", "m", "v"))
        if s["bits"] == 8:
            size = m - torch.where(m >= 128, 128.0, 0.0)
            m = torch.where(m >= 128, -1.0, 1.0) * (size * size) * q["m_unit"][:, None]
            v = (v * v) * q["v_unit"][:, None]
            v = v * v
        m = m * BETA1 + g * (1 - BETA1)
        v = v * BETA2 + (g * g) * (1 - BETA2)
        root = torch.sqrt(v)
        p = p * (1 - LR * DECAY) - (m * (LR / b1)) / (root * (1 / math.sqrt(b2)) + ADAM_EPS)
        q["p"].copy_(p)
        if s["bits"] == 32:
            q["m"].copy_(m)
            q["v"].copy_(v)
            got.update({"p%d" % i: q["p"], "m%d" % i: q["m"], "v%d" % i: q["v"]})
            continue
        chance = _plain_chance(q, step)
        q["m_unit"].copy_(m.abs().amax(1) * (1 / 127 ** 2))
        q["v_unit"].copy_(root.amax(1) * (1 / 255 ** 2))
        code = _plain_code(m.abs(), 127, q["m_unit"], chance, 1)
        value = torch.where(m < 0, -1.0, 1.0) * (code * code) * q["m_unit"][:, None]
        q["m"].copy_(code + 128 * ((m < 0) & (code > 0)))
        code = _plain_code(root, 255, q["v_unit"], chance, 2)
        code = torch.where((root > 0) & (code == 0), 1.0, code)   # a second moment of zero is none
        q["v"].copy_(code)
        back = (code * code) * q["v_unit"][:, None]
        got.update({"p%d" % i: q["p"], "m%d" % i: value.bfloat16().view(-1), "v%d" % i: (back * back).bfloat16().view(-1)})
    return got


# ---- one pass --------------------------------------------------------------------------------

def run(state):
    s = state
    if s["kind"] == "adamw":
        s["step"] += 1
    if not own:
        return {"norm": _plain_norm, "draws": _plain_draws, "adamw": _plain_adamw}[s["kind"]](s)
    import paper_2402_05396_amd as T
    if s["kind"] == "norm":
        if not s["train"]:
            return {"out": T.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)}
        out, stats = T.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, want_stats=True)
        dx, dweight, dbias = T.layer_norm_grad(s["dout"], s["x"], stats, s["weight"], s["bias"])
        return {"out": out, "dx": dx, "dweight": dweight, "dbias": dbias}
    if s["kind"] == "draws":
        action, logp = T.policy_draw(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], count=s["count"])
        return {"action": action, "logp": logp}
    T.adamw_step(s["params"], s["grads"], s["m"], s["v"], s["step"], lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY, units=s["units"] if s["bits"] == 8 else None)
    got = {}
    for i, q in enumerate(s["groups"]):
        m, v = q["m"], q["v"]
        if s["bits"] == 8:
            m, v = T.adamw_moments(m.view(-1), v.view(-1), (q["m_unit"], q["v_unit"]), dtype=torch.bfloat16)
        got.update({"p%d" % i: q["p"], "m%d" % i: m, "v%d" % i: v})
    return got


# ---- the definition, in 64 bits ----------------------------------------------------------------

def _exact_norm(s):
    x = s["x"].double().requires_grad_(s["train"])
    weight, bias = (s[n].double().requires_grad_(s["train"]) for n in ("weight", "bias"))
    spread, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    out = (x - mean) / (spread + EPS) ** 0.5 * weight + bias
    got = {"out": out.detach()}
    if s["train"]:
        got.update(zip(("dx", "dweight", "dbias"), torch.autograd.grad(out, (x, weight, bias), s["dout"].double())))
    return got


def _exact_draws(s):
    settings = _settings(s)
    actions, logps = [], []
    for i in range(0, s["rows"], 128):
        x = s["logits"][i:i + 128].double()
        index = torch.arange(s["width"], device="cuda")
        if s["count"] is not None:
            x = x.masked_fill(index >= s["count"][i:i + 128, None], -math.inf)
        t, k, p, least = (y[i:i + 128] for y in settings)
        order = torch.argsort(-x, dim=1, stable=True)
        rank = torch.empty_like(order).scatter_(1, order, index.expand_as(order).contiguous())
        greedy, none = t == 0, (x == -math.inf).all(1, keepdim=True)
        share = torch.softmax((x / torch.where(greedy, 1.0, t)).masked_fill((k > 0) & (rank >= k), -math.inf).masked_fill(greedy & (rank > 0), -math.inf), 1).nan_to_num(0.0)
        falling = share.gather(1, order)
        ahead = (falling.cumsum(1) - falling).gather(1, rank)
        out = ((p < 1) & (ahead >= p)) | (share < least * share.amax(1, keepdim=True))
        share = share.masked_fill(out & (rank > 0), 0.0)
        upto = (share / share.sum(1, keepdim=True)).cumsum(1)
        which = torch.stack([(upto <= s["uniform"][i:i + 128, j:j + 1].double()).sum(1) for j in range(s["picks"])], 1).clamp(max=s["width"] - 1)
        logp = torch.log_softmax(x, 1).gather(1, which)
        actions.append(which.masked_fill(none, -1).int())
        logps.append(logp.masked_fill(none, 0.0))
    return {"action": torch.cat(actions), "logp": torch.cat(logps)}


def _exact_words(count, block, number, step):
    """float64 [blocks, count * 8]: chances of a tensor's pieces, by products of 16-bit halves."""
    def product(a, x):   # (high, low) word of a 32-bit constant and 32-bit numbers
        a0, a1, x0, x1 = a & 0xFFFF, a >> 16, x & 0xFFFF, x >> 16
        middle = a1 * x0 + (a0 * x0 >> 16)
        other = a0 * x1 + (middle & 0xFFFF)
        return a1 * x1 + (middle >> 16) + (other >> 16), (other & 0xFFFF) << 16 | a0 * x0 & 0xFFFF

    x0 = block[:, None] * count + torch.arange(count, device="cuda")
    x1, x2, x3 = number[:, None] + 0 * x0, 0 * x0 + step, 0 * x0 + TAG
    for i in range(10):
        h0, l0 = product(0xD2511F53, x0)
        h2, l2 = product(0xCD9E8D57, x2)
        x0, x1, x2, x3 = h2 ^ x1 ^ (i * 0x9E3779B9 & 0xFFFFFFFF), l2, h0 ^ x3 ^ (i * 0xBB67AE85 & 0xFFFFFFFF), l0
    parts = [h for x in (x0, x1, x2, x3) for h in (x % 65536, x // 65536)]
    return ((torch.stack(parts, 2).double() + 0.5) / 65536).flatten(1)


def _exact_adamw(s):
    got, t = {}, s["step"] + 1
    for i, q in enumerate(s["groups"]):
        m, v = q["m"].double(), q["v"].double()
        if s["bits"] == 8:
            sign = 1 - 2 * (q["m"] // 128).double()
            m = sign * (q["m"] % 128).double() ** 2 * q["m_unit"].double()[:, None]
            v = (v ** 2 * q["v_unit"].double()[:, None]) ** 2
        g = q["g"].double()
        m = m + (1 - BETA1) * (g - m)
        v = v + (1 - BETA2) * (g ** 2 - v)
        p = q["p"].double()
        p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + ADAM_EPS)
        if s["bits"] == 8:
            u = _exact_words(BLOCK // 8, q["place"], q["number"], t)
            for name, x, most in (("m", m.abs(), 127), ("v", v, 255)):
                power = 2 if name == "m" else 4
                unit = x.amax(1, keepdim=True) / most ** power
                y = torch.where(unit > 0, x / unit, 0.0)
                low = (y ** (1 / power)).floor().clamp(max=most - 1)
                code = low + (y - low ** power > u * ((low + 1) ** power - low ** power))
                if name == "v":
                    code = torch.where((x > 0) & (code == 0), 1.0, code)
                    v = code ** 4 * unit
                else:
                    m = torch.sign(m) * code ** 2 * unit
            m, v = m.view(-1), v.view(-1)
        got.update({"p%d" % i: p, "m%d" % i: m, "v%d" % i: v})
    return got


def exact(case, seed):
    return {"norm": _exact_norm, "draws": _exact_draws, "adamw": _exact_adamw}[case["kind"]](prepare(case, seed))
