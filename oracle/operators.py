"""Attention to states of another length, the bias by distance, the clipped policy loss, layer norm, a policy's draws and the AdamW
step from their definitions, in 64 bits on the CPU, with how far a result in fewer bits may be off.

The bounds follow from the roundings that the operators say they make. u is half the spacing of the element type above 1 (2^-24,
2^-11, 2^-8), `tiny` half its spacing at 0. Softmax weights, their gradients dx and
outputs are each rounded once to the type: u of the value plus `tiny`. Everything else is in 32 bits: a sum of n terms is off by at
most n 2^-24 of the sum of their magnitudes, and an error d in a score changes a weight by a factor 1 + 2 d.
"""
import numpy as np

U = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 0.0, "float16": 2.0 ** -25, "bfloat16": 0.0}
E32 = 2.0 ** -24
END32 = 2.0 ** -125   # 32-bit numbers end at 2^-126: a smaller weight, or product with one, may be 0


def buckets(bounds, query_pos, key_pos):
    """[queries], [keys] -> [queries, keys]: how many bounds are at most the distance (Python integers: no overflow)."""
    apart = np.array([[int(a) - int(b) for b in key_pos] for a in query_pos], dtype=object).reshape(len(query_pos), len(key_pos))
    out = np.zeros(apart.shape, np.int64)
    for bound in bounds:
        out += (apart >= int(bound)).astype(np.int64)
    return out


def attention(q, k, v, kind, lengths=None, mask=None, table=None, bucket=None, scale=None, dout=None, lifted=False):
    """q [B, Lq, H, d], k, v [B, Lk, Hk, d] float64; bucket: a list of [Lq, Lk] for each batch entry. -> (results, bounds): dicts of
    out, and with `dout` dq, dk, dv, dtable. lifted: the bounds of an operator that multiplies dx by a power of two before it rounds it to
    float16, for each row of dq and each state of dk so that the largest comes to 2^7 at least: not `tiny` each, but 2^-7 `tiny` of the largest."""
    B, Lq, H, d = q.shape
    Lk, Hk = k.shape[1:3]
    g = H // Hk
    scale = d ** -0.5 if scale is None else scale
    u, tiny = U[kind], TINY[kind]
    u16 = 0.0 if kind == "float32" else u          # what is rounded to the type between the products
    res = {n: np.zeros(s) for n, s in (("out", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", v.shape))}
    off = {n: np.zeros_like(x) for n, x in res.items()}
    if table is not None:
        res["dtable"], off["dtable"] = np.zeros_like(table), np.zeros_like(table)
    for b in range(B):
        seen = np.ones(Lk, bool) if mask is None else np.asarray(mask[b]).astype(bool)
        if lengths is not None:
            seen = seen & (np.arange(Lk) < min(max(int(lengths[b]), 0), Lk))
        at = np.nonzero(seen)[0]
        if not len(at):
            continue
        for h in range(H):
            Q, K, V = q[b, :, h], k[b, at, h // g], v[b, at, h // g]
            x = Q @ K.T * scale
            ex = (d + 8) * E32 * scale * (np.abs(Q) @ np.abs(K).T)
            if table is not None:
                bias = table[h][bucket[b][:, at]]
                x = x + bias
                ex = ex + 4 * E32 * np.where(np.isfinite(bias), np.abs(bias) + np.abs(x), 0.0)
            top = x.max(1, keepdims=True)
            real = np.isfinite(top) | np.isnan(top)
            with np.errstate(invalid="ignore"):
                e = np.where(real, np.exp(x - np.where(real, top, 0)), 0.0)
            s = e.sum(1, keepdims=True)
            p = e / np.where(s == 0, 1, s)
            far = np.where(p > 0, np.abs(x - np.where(real, top, 0)), 0.0)
            most = ex.max(1, keepdims=True)
            ep = p * (2 * (ex + most) + (far + len(at) + 32) * E32) + END32      # a weight in 32 bits
            o = p @ V
            res["out"][b, :, h] = o
            eo = ep @ np.abs(V) + (len(at) + 8) * E32 * (p @ np.abs(V)) + (u16 * p) @ np.abs(V) + tiny * 2.0 ** -14 * np.abs(V).sum(0)
            off["out"][b, :, h] = eo + u * (np.abs(o) + eo) + tiny
            if dout is None:
                continue
            Y = dout[b, :, h]
            dp, t = Y @ V.T, (Y * o).sum(1, keepdims=True)
            dx = p * (dp - t)
            et = (np.abs(Y) * off["out"][b, :, h]).sum(1, keepdims=True) + d * E32 * (np.abs(Y) * np.abs(o)).sum(1, keepdims=True)
            edx = ep * np.abs(dp - t) + p * ((d + 4) * E32 * (np.abs(Y) @ np.abs(V).T) + et) + 4 * E32 * np.abs(dx) + END32
            rdx = edx + u16 * np.abs(dx)                                           # where it enters a product
            rdq, rdk = rdx + (tiny if u16 else 0.0), rdx + (tiny if u16 else 0.0)
            if lifted and u16:                                                     # a state has one factor for all heads that share it
                rdq = rdx + 2.0 ** -7 * tiny * (rdx + np.abs(dx)).max(1, keepdims=True)
                largest, weights = (0.0, 0.0) if h % g == 0 else (largest, weights)
                largest, weights, rdk = np.maximum(largest, (rdx + np.abs(dx)).max(0)), weights + np.abs(Q).sum(0), rdx
                if h % g == g - 1:
                    off["dk"][b, at, h // g] += scale * 2.0 ** -7 * tiny * largest[:, None] * weights
            n = (Lq * g + len(at) + 8) * E32
            for name, of, value, err in (("dq", (b, slice(None), h), scale * dx @ K, scale * (rdq @ np.abs(K) + n * np.abs(dx) @ np.abs(K))),):
                res[name][of] += value
                off[name][of] += err
            res["dk"][b, at, h // g] += scale * dx.T @ Q
            off["dk"][b, at, h // g] += scale * (rdk.T @ np.abs(Q) + n * np.abs(dx).T @ np.abs(Q))
            res["dv"][b, at, h // g] += p.T @ Y
            off["dv"][b, at, h // g] += (ep + (u16 + n) * p).T @ np.abs(Y) + (tiny * 2.0 ** -14 * np.abs(Y).sum(0) if u16 else 0.0)
            if table is not None:
                for i in range(table.shape[1]):
                    here = bucket[b][:, at] == i
                    res["dtable"][h, i] += dx[here].sum()
                    off["dtable"][h, i] += (edx + (B * Lq * g + len(at)) * E32 * np.abs(dx))[here].sum()
    for n in ("dq", "dk", "dv", "dtable"):
        if n in res:
            off[n] = off[n] + u * (np.abs(res[n]) + off[n]) + tiny
    keep = ["out"] + (["dq", "dk", "dv"] + (["dtable"] if table is not None else []) if dout is not None else [])
    return {n: res[n] for n in keep}, {n: off[n] for n in keep}


def policy_loss(logits, actions, advantage, kind, old=None, ref=None, count=None, weight=None, low=0.2, high=0.2, kl=0.0):
    """logits float64 [R, W]; actions int [R, n] -> (results, bounds) of loss, logp, grad."""
    R, W = logits.shape
    n = actions.shape[1]
    u, tiny = U[kind], TINY[kind]
    loss, logp, grad = np.zeros((R, n)), np.zeros((R, n)), np.zeros((R, W))
    eloss, elogp, egrad = np.zeros((R, n)), np.zeros((R, n)), np.zeros((R, W))
    for r in range(R):
        c = W if count is None else min(max(int(count[r]), 0), W)
        if not c:
            continue
        x = logits[r, :c]
        top = x.max()
        e = np.exp(x - top)
        s = e.sum()
        p = e / s
        ep = p * ((c + 16) * E32 + 4 * E32 * np.abs(np.where(p > 0, x - top, 0.0))) + END32
        slopes, eslopes = 0.0, 0.0
        extra, eextra = np.zeros(c), np.zeros(c)
        for j in range(n):
            a = int(actions[r, j])
            if not 0 <= a < c:
                continue
            l = x[a] - top - np.log(s)
            el = (c + 16) * E32 + 4 * E32 * (abs(x[a] - top) + abs(np.log(s)) + abs(x[a]))
            A, w = float(advantage[r, j]), 1.0 if weight is None else float(weight[r, j])
            logp[r, j], elogp[r, j] = l, el
            if w == 0:
                continue
            ratio = 1.0 if old is None else np.exp(l - float(old[r, j]))
            eratio = 0.0 if old is None else ratio * (2 * el + 4 * E32 * (1 + abs(l) + abs(float(old[r, j]))))
            whole = ratio * A
            cut = whole if old is None else min(max(ratio, 1 - low), 1 + high) * A
            y, dy = -min(whole, cut), -whole if whole <= cut else 0.0
            ey = (eratio + 4 * E32 * (1 + ratio)) * abs(A)
            edy = ey if old is None or min(abs(ratio - 1 + low), abs(ratio - 1 - high)) > eratio + 4 * E32 else abs(whole) + ey   # a ratio at a bound may fall to either side
            if ref is not None:
                t = float(ref[r, j]) - l
                et = np.exp(t) * (2 * el + 4 * E32 * (1 + abs(t) + abs(float(ref[r, j])))) + 8 * E32 * (np.exp(t) + abs(t) + 1)
                y, dy, ey, edy = y + kl * (np.exp(t) - t - 1), dy + kl * (1 - np.exp(t)), ey + kl * (et + el), edy + kl * et
            loss[r, j], eloss[r, j] = w * y, abs(w) * (ey + 4 * E32 * abs(y))
            slopes, eslopes = slopes + w * dy, eslopes + abs(w) * (edy + (n + 4) * E32 * abs(dy))
            extra[a] += w * dy
            eextra[a] += abs(w) * (edy + (n + 4) * E32 * abs(dy))
        grad[r, :c] = extra - slopes * p
        egrad[r, :c] = eextra + eslopes * p + abs(slopes) * (ep + 4 * E32 * p) + 2 * E32 * (np.abs(extra) + abs(slopes) * p)
    egrad = egrad + u * (np.abs(grad) + egrad) + tiny
    return {"loss": loss, "logp": logp, "grad": grad}, {"loss": eloss, "logp": elogp, "grad": egrad}


def layer_norm(x, kind, weight=None, bias=None, eps=1e-5, dout=None, kept=None, depth=None):
    """x, dout float64 [R, W]; kept: the weights' kind, kind unless given -> (results, bounds) of out, the statistics mean and rstd [R, 1] and, with `dout`,
    dx, dweight, dbias. The operator's sums are in 32 bits; out and the gradients are rounded to their types once. depth: how many additions
    a number goes through at most, in a row's sums and in those over the rows (unless given: as many as there are numbers, which says least)."""
    R, W = x.shape
    across, down = (W, R) if depth is None else depth
    u, tiny = U[kind], TINY[kind]
    u2, tiny2 = U[kept or kind], TINY[kept or kind]
    w = np.ones(W) if weight is None else weight
    b = np.zeros(W) if bias is None else bias
    mean = x.mean(1, keepdims=True)
    away = x - mean
    em = (across + 4) * E32 * np.abs(x).mean(1, keepdims=True) + E32 * np.abs(mean)
    ea = em + E32 * np.abs(away)
    var = (away ** 2).mean(1, keepdims=True) + eps
    evar = (2 * np.abs(away) * ea + ea ** 2).mean(1, keepdims=True) + (across + 8) * E32 * var
    rstd = var ** -0.5
    part = np.minimum(evar / var, 0.99)
    er = rstd * ((1 - part) ** -0.5 - 1 + 4 * E32)
    xhat = away * rstd
    ex = ea * (rstd + er) + np.abs(away) * er + 2 * E32 * np.abs(xhat)
    out = xhat * w + b
    eo = ex * np.abs(w) + 4 * E32 * (np.abs(xhat * w) + np.abs(b))
    res, off = {"out": out, "mean": mean, "rstd": rstd}, {"out": eo + u * (np.abs(out) + eo) + tiny, "mean": em, "rstd": er}
    if dout is None:
        return res, off
    g = dout * w
    s, t = g.mean(1, keepdims=True), (g * xhat).mean(1, keepdims=True)
    es = (across + 6) * E32 * np.abs(g).mean(1, keepdims=True)
    et = (np.abs(g) * ex).mean(1, keepdims=True) + (across + 8) * E32 * np.abs(g * xhat).mean(1, keepdims=True)
    inner = g - s - xhat * t
    ei = 4 * E32 * (np.abs(g) + np.abs(s) + np.abs(xhat * t)) + es + ex * (np.abs(t) + et) + np.abs(xhat) * et
    dx = rstd * inner
    ed = (rstd + er) * ei + er * np.abs(inner) + 2 * E32 * np.abs(dx)
    dweight, dbias = (dout * xhat).sum(0), dout.sum(0)
    ew = (np.abs(dout) * ex).sum(0) + (down + 8) * E32 * np.abs(dout * xhat).sum(0)
    eb = (down + 8) * E32 * np.abs(dout).sum(0)
    res.update(dx=dx, dweight=dweight, dbias=dbias)
    off.update(dx=ed + u * (np.abs(dx) + ed) + tiny, dweight=ew + u2 * (np.abs(dweight) + ew) + tiny2, dbias=eb + u2 * (np.abs(dbias) + eb) + tiny2)
    return res, off


def policy_draw(logits, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, count=None):
    """logits, uniform float64 [R, W], [R, n]; settings numbers or arrays [R], as the operator has them (in 32 bits) -> (actions, logp, how far logp
    may be off, sure). sure: the draw is further from every border (of top-p's share, min_p's weight, the running sum) than weights that are whole
    multiples of 2^-43, off by another 2^-41 of their own, could move it."""
    R, W = logits.shape
    n = uniform.shape[1]
    of = lambda x: np.broadcast_to(np.asarray(x, np.float64), (R,))
    temperature, top_k, top_p, min_p = of(temperature), of(top_k), of(top_p), of(min_p)
    actions, logp, off, sure = np.full((R, n), -1), np.zeros((R, n)), np.zeros((R, n)), np.ones((R, n), bool)
    for r in range(R):
        c = W if count is None else min(max(int(count[r]), 0), W)
        x = logits[r, :c]
        if not c or (np.isneginf(x).all()):
            continue
        if np.isnan(x).any() or np.isposinf(x).any():
            logp[r] = np.nan
            continue
        top = x.max()
        order = np.argsort(-x, kind="stable")
        w = np.zeros(c)
        if temperature[r] > 0:
            w = np.exp((x - top) / temperature[r])
            w[np.isneginf(x)] = 0
        else:
            w[order[0]] = 1
        rounded = (w != 0) & (w != 1)   # the others, and their sums, are exact on either side
        slack = lambda s: min(s, w[rounded].sum()) * 2.0 ** -41 + rounded.sum() * 2.0 ** -43
        clear = lambda margin, s: margin > slack(s) or slack(s) == 0
        k = min(int(top_k[r]), c) if top_k[r] > 0 else c
        best, there = order[:k], w[order[:k]]
        before, whole = np.cumsum(there) - there, there.sum()
        keep, certain = np.zeros(c, bool), True
        stays = np.ones(k, bool)
        if top_p[r] < 1:
            stays = before < top_p[r] * whole
            margin = np.abs(before - top_p[r] * whole)[1:]
            certain = len(margin) == 0 or clear(margin.min(), whole)
        if min_p[r] > 0:
            margin = np.abs(there - min_p[r])[1:][there[1:] != 1]
            certain = certain and (len(margin) == 0 or clear(margin.min(), 1.0))
            stays &= there >= min_p[r]
        stays[0] = True
        keep[best] = stays
        running = np.cumsum(np.where(keep, w, 0.0))
        last = np.nonzero(np.where(keep, w, 0.0) > 2.0 ** -45)[0][-1]
        s = np.exp(x - top).sum()
        for j in range(n):
            place = min(max(uniform[r, j], 0.0), 1.0) * running[-1]
            a = min(int((running <= place).sum()), last)
            actions[r, j] = a
            away = [abs(y - place) for y in (running[a], running[a - 1] if a else np.inf)]
            sure[r, j] = certain and (keep.sum() == 1 or uniform[r, j] == 0 or clear(min(away), running[-1]))
            logp[r, j] = x[a] - top - np.log(s)
            off[r, j] = (c + 16) * E32 + 4 * E32 * (abs(x[a] - top) + abs(np.log(s)) + abs(x[a]))
    return actions, logp, off, sure


def philox(counter, key):
    """Philox4x32-10: counter, four uint32 arrays; key, two numbers -> four uint32 arrays."""
    c, k = [np.asarray(x, np.uint64) for x in counter], [int(x) for x in key]
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> shift) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> shift) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return [x.astype(np.uint32) for x in c]


def adamw_chance(n, number, step, seed):
    """float64 [n]: what an 8-bit moment's place between its two codes is compared with."""
    piece = np.arange((n + 7) // 8, dtype=np.uint64)
    same = lambda x: np.full(piece.shape, x & 0xFFFFFFFF, np.uint64)
    words = philox((piece & np.uint64(0xFFFFFFFF), same(number), same(step), same(0x4144414D)), (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
    halves = np.stack([h for x in words for h in (x & np.uint32(0xFFFF), x >> np.uint32(16))], 1).reshape(-1)[:n]
    return (halves.astype(np.float64) + 0.5) / 65536


def adamw_decode(m, v, m_unit, v_unit):
    """Codes and units -> moments, in 64 bits."""
    at = np.arange(len(m)) // 256
    m, v = m.astype(np.int64), v.astype(np.float64)
    return np.where(m >= 128, -1.0, 1.0) * (m % 128) ** 2 * m_unit.astype(np.float64)[at], (v ** 2 * v_unit.astype(np.float64)[at]) ** 2


def adamw(p, g, m, v, kind, step, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.01, scale=1.0):
    """float64 arrays -> (results, bounds) of p, m, v. Multipliers are rounded to 32 bits, as every product and sum is."""
    g = g * scale
    eg = E32 * np.abs(g) if scale != 1.0 else 0.0
    m2, v2 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    em = 4 * E32 * (np.abs(beta1 * m) + np.abs((1 - beta1) * g)) + (1 - beta1) * eg + END32
    ev = 6 * E32 * v2 + 2 * (1 - beta2) * np.abs(g) * eg + END32
    c1, c2 = 1 - beta1 ** step, 1 - beta2 ** step
    root = np.sqrt(v2)
    eroot = np.sqrt(v2 + ev) - root + 2 * E32 * root
    den = root / np.sqrt(c2) + eps
    eden = eroot / np.sqrt(c2) + 4 * E32 * den
    with np.errstate(divide="ignore", invalid="ignore"):
        move = lr / c1 * m2 / den
        emove = lr / c1 * em / den + np.abs(move) * (eden / np.maximum(den - eden, 1e-300) + 10 * E32)
    out = p * (1 - lr * decay) - move
    ep = 3 * E32 * np.abs(p) + emove + 2 * E32 * np.abs(move) + END32
    return {"p": out, "m": m2, "v": v2}, {"p": ep + U[kind] * (np.abs(out) + ep) + TINY[kind], "m": em, "v": ev}


def adamw_codes(x, chance, quad):
    """Magnitudes of one block (64 bits), their chances -> (codes, sure, unit): quad: x = (unit c^2)^2, else unit c^2. sure: the code is the same where x is off by
    20 * 2^-24 of itself and of the block's largest."""
    power, most = (4, 255) if quad else (2, 127)
    largest = x.max() if len(x) else 0.0
    if largest == 0:
        return np.zeros(len(x), np.int64), np.ones(len(x), bool), 0.0
    y = x / largest * float(most) ** power
    c = np.minimum(np.floor(y ** (1 / power)), most - 1)
    low, high = c ** power, (c + 1) ** power
    place = (y - low) / (high - low)
    codes = (c + (place > chance)).astype(np.int64)
    if quad:
        codes[(x > 0) & (codes == 0)] = 1
    slack = 40 * E32 * y / (high - low)
    sure = np.abs(place - chance) > slack
    return codes, sure, largest
