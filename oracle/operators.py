"""Attention to states of another length, the bias by distance and the clipped policy loss from their definitions, in 64 bits on
the CPU, with how far a result in fewer bits may be off.

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
