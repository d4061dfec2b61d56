"""The AdamW step, moments in 32 and in 8 bits, against its definition in 64 bits (GPU), the oracle against other forms of it (CPU)."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2402_05396_amd as T
from oracle import operators as O

KINDS = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
gpu = pytest.mark.gpu
SIZES = [1, 3, 255, 256, 257, 1000, 4095, 4096, 4097, 12_345, 100_001]


class Absent:
    def __getattr__(self, name):
        return lambda *a: None


def _case(bits, sizes=SIZES, kind="float32", grads=None, seed=0, padding=0):
    """Tensors of these sizes and moments some steps old, on the GPU; `padding` elements lie before each in its memory."""
    g = torch.Generator().manual_seed(seed)
    rnd = lambda n: torch.randn(n, generator=g)
    place = lambda t: torch.cat([torch.zeros(padding, dtype=t.dtype), t]).cuda()[padding:]
    c = dict(params=[], grads=[], m=[], v=[], units=None if bits == 32 else ([], []))
    for n in sizes:
        size = torch.exp(rnd(-(-n // 256)) * 2 - 6).repeat_interleave(256)[:n]
        c["params"].append(place((rnd(n) * 0.1).to(KINDS[kind])))
        c["grads"].append(place((rnd(n) * size).to(KINDS[grads or kind])))
        if bits == 32:
            c["m"].append(place(0.3 * rnd(n) * size))
            c["v"].append(place(((0.5 + torch.rand(n, generator=g)) * size) ** 2))
        else:
            blocks = -(-n // 256)
            cv = torch.randint(0, 256, (n,), generator=g)
            c["v"].append(place(cv.to(torch.uint8)))
            c["m"].append(place(((cv * torch.rand(n, generator=g) * (127 / 255)).long() + 128 * torch.randint(0, 2, (n,), generator=g)).to(torch.uint8)))
            c["units"][0].append(0.8 * size[::256].contiguous().cuda() / 127 ** 2)
            c["units"][1].append(2 * size[::256].contiguous().cuda() / 255 ** 2)
            assert c["units"][0][-1].numel() == blocks
    return c


def _copy(c):
    return {n: x if x is None else tuple([t.clone() for t in y] for y in x) if n == "units" else [None if t is None else t.clone() for t in x] for n, x in c.items()}


def _step(c, step, **more):
    T.adamw_step(c["params"], c["grads"], c["m"], c["v"], step, units=c["units"], **more)


def _arr(t):
    return t.double().cpu().numpy() if t.dtype.is_floating_point else t.cpu().numpy()


def _check(before, after, kind, step, seed=0, scale=1.0, **more):
    for i, (p, g, m, v) in enumerate(zip(*(before[n] for n in ("params", "grads", "m", "v")))):
        new_m, new_v = _arr(after["m"][i]), _arr(after["v"][i])
        if g is None:
            assert torch.equal(after["params"][i], p) and torch.equal(after["m"][i], m) and torch.equal(after["v"][i], v)
            continue
        old_m, old_v = _arr(m), _arr(v)
        if before["units"]:
            units = [_arr(u[i]) for u in before["units"]]
            old_m, old_v = O.adamw_decode(old_m, old_v, *units)
            # decoded in 32 bits: two roundings of m, four of v
            decoded = 2 * O.E32 * np.abs(old_m), 4 * O.E32 * old_v
        want, off = O.adamw(_arr(p), _arr(g), old_m, old_v, kind, step, scale=scale, **more)
        far = np.abs(_arr(after["params"][i]) - want["p"])
        if before["units"] is None:
            assert (far <= off["p"]).all(), (i, float((far - off["p"]).max()))
            assert (np.abs(new_m - want["m"]) <= off["m"]).all() and (np.abs(new_v - want["v"]) <= off["v"]).all(), i
            continue
        # the moments that the parameter saw were off by the decoding besides: of the update m / sqrt(v), as much as it moves per part of either
        move = np.abs(want["p"] - _arr(p) * (1 - more.get("lr", 1e-3) * more.get("decay", 0.01)))
        assert (far <= off["p"] + 4 * O.E32 * move + more.get("lr", 1e-3) / (1 - 0.9 ** step) * decoded[0] / (np.sqrt(want["v"] / (1 - 0.999 ** step)) + 1e-8)).all(), i
        chance, n = O.adamw_chance(len(new_m), i, step, seed), len(new_m)
        for name, codes, unit, quad in (("m", new_m & 127, _arr(after["units"][0][i]), False), ("v", new_v, _arr(after["units"][1][i]), True)):
            for b in range(-(-n // 256)):
                of = slice(256 * b, min(n, 256 * b + 256))
                x = np.abs(want[name][of])
                exact, sure, largest = O.adamw_codes(x, chance[of], quad)
                slack = np.abs(off[name][of]).max() + 8 * O.E32 * largest + (decoded[0][of].max() if name == "m" else decoded[1][of].max())
                most = (255.0 ** 2 * unit[b]) ** 2 if quad else 127.0 ** 2 * unit[b]
                assert abs(most - largest) <= slack, (i, b)
                # m is a sum of terms of either sign, off by roundings of the terms: only where it is not much less than those is its code certain
                if not quad:
                    with np.errstate(divide="ignore", invalid="ignore"):
                        y = x / largest * 127 ** 2
                        c = np.minimum(np.floor(np.sqrt(y)), 126)
                        sure &= np.abs((y - c * c) / (2 * c + 1) - chance[of]) > 127 ** 2 / largest * (off[name][of] + decoded[0][of]) / (2 * c + 1) + 40 * O.E32 * y / (2 * c + 1)
                assert (codes[of] == exact)[sure].all(), (i, b, name)
                assert sure.mean() > 0.95 or len(sure) < 30
                assert (np.abs(codes[of].astype(np.int64) - exact) <= 1).all()
        sure = np.abs(want["m"]) > off["m"] + decoded[0]
        assert ((new_m >> 7 == 1) == (want["m"] < 0))[sure & (new_m & 127 != 0)].all()


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind,grads", [("float32", "float32"), ("float32", "bfloat16"), ("float32", "float16"), ("bfloat16", "bfloat16"), ("float16", "float16"), ("bfloat16", "float32"), ("float16", "float32"),
                                        ("float16", "bfloat16"), ("bfloat16", "float16")])
def test_against_64_bits(bits, kind, grads):
    for step, padding, more in ((1, 0, {}), (7, 1, dict(lr=0.02, weight_decay=0.0)), (100_000, 3, dict(lr=1e-4, weight_decay=0.1))):
        before = _case(bits, kind=kind, grads=grads, seed=step, padding=padding)
        after = _copy(before) if not padding else before
        if padding:
            before = _copy(after)
        _step(after, step, seed=step * 2 ** 33 + 5, **more)
        given = {"lr": more.get("lr", 1e-3), "decay": more.get("weight_decay", 0.01)}
        _check(before, after, kind, step, seed=step * 2 ** 33 + 5, **given)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(bits):
    """More than a launch takes, some empty, some without a gradient; each keeps its place in the list."""
    rng = np.random.default_rng(0)
    before = _case(bits, sizes=[int(n) for n in rng.integers(1, 6000, 150)] + [300_000], seed=1)
    for i in (0, 5, 60, 149):
        before["grads"][i] = None
    for i in (3, 70):
        for n in ("params", "grads", "m", "v"):
            before[n][i] = before[n][i][:0]
        if before["units"]:
            for u in before["units"]:
                u[i] = u[i][:0]
    after = _copy(before)
    _step(after, 3, seed=11)
    for i in (3, 70):
        for n in ("params", "grads", "m", "v"):
            before[n][i] = after[n][i] = torch.zeros(1, device="cuda") if n != "grads" else None
    _check(before, after, "float32", 3, seed=11, lr=1e-3, decay=0.01)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_what_lies_beside_a_tensor_is_left(bits):
    for kind, n in (("float32", 257), ("bfloat16", 1001), ("float16", 4097), ("float32", 3)):
        whole = {name: torch.full((n + 12,), 7, dtype=dtype, device="cuda") for name, dtype in
                 (("p", KINDS[kind]), ("g", KINDS[kind]), ("m", torch.uint8 if bits == 8 else torch.float32), ("v", torch.uint8 if bits == 8 else torch.float32))}
        units = None if bits == 32 else tuple([torch.ones(-(-n // 256) + 4, device="cuda")] for _ in range(2))
        inner = None if bits == 32 else tuple([u[0][2:-2]] for u in units)
        T.adamw_step(*([whole[name][5:n + 5]] for name in "pgmv"), 2, lr=1.0, units=inner)   # (far more than a rounding of 7)
        for t in whole.values():
            assert (t[:5] == 7).all() and (t[n + 5:] == 7).all()
        assert (whole["p"][5:n + 5] != 7).any() and (whole["g"] == 7).all()
        if units:
            assert all((u[0][:2] == 1).all() and (u[0][-2:] == 1).all() for u in units)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_numbers_on_the_device_graph_and_halves(bits, monkeypatch):
    """Step, rate and the gradients' factor as tensors: a captured step goes on as the eager one does."""
    start = _case(bits, seed=3)
    step, lr, scale = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 1e-2, device="cuda"), torch.full((1,), 0.5, device="cuda")
    a, b = _copy(start), _copy(start)
    _step(_copy(start), 1)
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        _step(a, step, lr=lr, grad_scale=scale, seed=4)
    with torch.cuda.graph(second, pool=graph.pool()):
        step.add_(1)
        _step(a, step, lr=lr, grad_scale=scale, seed=4)
    for i in range(1, 6):
        for g in a["grads"]:
            g.mul_(0.9)
        (graph if i % 2 else second).replay()
        torch.cuda.synchronize()
        for g in b["grads"]:
            g.mul_(0.9)
        c = _copy(b)
        with monkeypatch.context() as m:
            m.setattr(T, "_native", Absent())
            _step(c, torch.tensor([i], device="cuda"), lr=torch.full((), 1e-2, device="cuda"), grad_scale=scale, seed=4)
        _step(b, torch.tensor([i], device="cuda"), lr=lr, grad_scale=scale, seed=4)
        for n in ("params", "m", "v"):
            assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(a[n], b[n], c[n])), (i, n)
    # numbers of the host's: a rate of 64 bits differs from one of 32 in its last places
    d = _copy(start)
    for g in d["grads"]:
        g.mul_(0.9)
    before = _copy(d)
    _step(d, 1, lr=float(np.float32(1e-2)), grad_scale=scale, seed=4)
    _check(before, d, "float32", 1, seed=4, scale=0.5, lr=float(np.float32(1e-2)), decay=0.01)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_factor_of_nan_changes_nothing(bits):
    before = _case(bits, seed=5)
    after = _copy(before)
    _step(after, 9, grad_scale=torch.full((1,), float("nan"), device="cuda"))
    for n in ("params", "m", "v"):
        assert all(torch.equal(x, y) for x, y in zip(before[n], after[n]))
    if bits == 8:
        assert all(torch.equal(x, y) for u, w in zip(before["units"], after["units"]) for x, y in zip(u, w))


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("number", [0, -3])
def test_a_step_on_the_device_below_1_changes_nothing(number, bits):
    before = _case(bits, seed=5)
    after = _copy(before)
    _step(after, torch.tensor([number], device="cuda"))
    for n in ("params", "m", "v"):
        assert all(torch.equal(x, y) for x, y in zip(before[n], after[n]))
    if bits == 8:
        assert all(torch.equal(x, y) for u, w in zip(before["units"], after["units"]) for x, y in zip(u, w))


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_finite(bits):
    before = _case(bits, sizes=[1000], seed=6)
    before["grads"][0][[3, 700]] = torch.tensor([float("nan"), float("inf")], device="cuda")
    after = _copy(before)
    _step(after, 4)
    p = after["params"][0]
    assert torch.isnan(p[[3, 700]]).all() and torch.isnan(p).sum() == 2
    if bits == 32:
        m, v = after["m"][0], after["v"][0]
        assert torch.isnan(m[3]) and torch.isinf(v[700]) and torch.isfinite(m).sum() == 998 == torch.isfinite(v).sum()
    else:   # a unit has 256 elements
        m, v = T.adamw_moments(after["m"][0], after["v"][0], (after["units"][0][0], after["units"][1][0]))
        for x in (m, v):
            assert torch.isnan(x[:256]).all() and torch.isnan(x[512:768]).all() and torch.isfinite(x[256:512]).all() and torch.isfinite(x[768:]).all()


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_moments_of_zero_and_tiny_ones(bits):
    params = [torch.ones(600, device="cuda") for _ in range(4)]
    grads = [torch.zeros(600, device="cuda"), torch.full((600,), 1e-30, device="cuda"), torch.full((600,), 1e-18, device="cuda"), torch.full((600,), 1e15, device="cuda")]
    m, v, units = T.adamw_state(params, bits)
    for step in (1, 2, 3):
        T.adamw_step(params, grads, m, v, step, units=units, weight_decay=0.0, lr=0.01)
    assert torch.equal(params[0], torch.ones(600, device="cuda")) and all(torch.isfinite(p).all() for p in params)
    # equal gradients: steps of lr g / (|g| + eps); in 8 bits a unit's elements are all its largest, each a few roundings off
    for p, size in zip(params[2:], (1e-18 / (1e-18 + 1e-8), 1.0)):
        assert (p - (1 - 0.03 * size)).abs().max() <= 3 * 0.01 * 64 * O.E32 + 4 * O.E32


@gpu
def test_second_moments_in_8_bits_follow_the_gradients():
    """A step with beta2 = 0.999 moves a second moment by a fraction of the distance of two codes. On average over 65536 elements it
    moves all the same. What the roundings add to a value is at most half of its distance d to the next code a step, independent: over n steps a
    standard deviation of at most d / 2 min(n, 500)^(1/2) for an element, the mean of N elements sqrt(N) times less; d is some 4 / 100 of a value at codes above 100."""
    n, steps = 65_536, 400
    g = torch.Generator("cuda").manual_seed(0)
    size = 0.5 + torch.rand(n, generator=g, device="cuda")
    p = [torch.zeros(n, device="cuda")]
    m, v, units = T.adamw_state(p, 8)
    for step in range(1, steps + 1):
        T.adamw_step(p, [size], m, v, step, lr=0.0, units=units, seed=3)
    got_m, got_v = T.adamw_moments(m[0], v[0], (units[0][0], units[1][0]))
    want = size.double() ** 2 * (1 - 0.999 ** steps)
    off = (got_v.double() / want - 1).mean().abs().item()
    assert off <= 6 * 0.02 * steps ** 0.5 / n ** 0.5 + steps * 8 * O.E32, off
    off = (got_m.double() / (size.double() * (1 - 0.9 ** steps)) - 1).mean().abs().item()
    # m: a tenth of it is new each step, so a code's distance, 2 / 60 at most, counts some 2.3 times
    assert off <= 6 * 2.3 / 60 / n ** 0.5 + 40 * O.E32, off


@gpu
@pytest.mark.parametrize("dtype", KINDS.values())
def test_moments_as_numbers(dtype):
    for n in (1, 7, 255, 256, 257, 5000):
        g = torch.Generator().manual_seed(n)
        m, v = (torch.randint(0, 256, (n,), generator=g).to(torch.uint8) for _ in range(2))
        units = [torch.rand(-(-n // 256), generator=g) * 1e-4 for _ in range(2)]
        got = T.adamw_moments(m.cuda(), v.cuda(), tuple(u.cuda() for u in units), dtype=dtype)
        want = O.adamw_decode(m.numpy(), v.numpy(), *(u.numpy() for u in units))
        kind = next(k for k, d in KINDS.items() if d == dtype)
        for x, y in zip(got, want):
            assert x.dtype == dtype and (np.abs(_arr(x) - y) <= (O.U[kind] + 5 * O.E32) * np.abs(y) + O.TINY[kind] + O.END32).all()


@gpu
def test_streams():
    before = _case(8, seed=7)
    want, got = _copy(before), _copy(before)
    _step(want, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _step(got, 2, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for n in ("params", "m", "v") for x, y in zip(want[n], got[n]))


@gpu
def test_refusals_of_the_binding():
    c = _case(32, sizes=[300, 40], seed=8)
    p, g, m, v = c["params"], c["grads"], c["m"], c["v"]
    T.adamw_step(p, g, m, v, 1)
    T.adamw_step(tuple(p), tuple(g), tuple(m), tuple(v), 1)
    kept = [t.clone() for t in p + m + v]
    two = torch.zeros(600, device="cuda")
    for error, args in ((TypeError, ([p[0].double(), p[1]], g, m, v, 1)), (TypeError, ([two[::2], p[1]], g, m, v, 1)), (TypeError, ([p[0].cpu(), p[1]], g, m, v, 1)),
                        (TypeError, (p, [g[0].double(), g[1]], m, v, 1)), (TypeError, (p, [two[::2], g[1]], m, v, 1)), (TypeError, (p, g, [m[0].half(), m[1]], v, 1)),
                        (TypeError, (p, g, m, [v[0].cpu(), v[1]], 1)), (ValueError, (p, g[:1], m, v, 1)), (ValueError, (p, [g[0][:299], g[1]], m, v, 1)),
                        (ValueError, (p, g, [m[0][:299], m[1]], v, 1)), (TypeError, (p, g, m, v, torch.ones(1, device="cuda")))):
        with pytest.raises(error):
            T.adamw_step(*args)
    for bad in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(weight_decay=-1.0), dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")), dict(step=0), dict(step=-3)):
        with pytest.raises(T.TaserError):
            T.adamw_step(p, g, m, v, **{"step": 1, **bad})
    # memory that is written, named twice
    for args in (([p[0], p[0]], [g[0], g[0]], [m[0], m[0].clone()], [v[0], v[0].clone()]), ([two[:300], two[290:330]], g, m, v), (p, g, m, [m[0], v[1]]), (p, [p[0], g[1]], m, v), (p, g, [g[0], m[1]], v)):
        with pytest.raises(T.TaserError, match="overlap"):
            T.adamw_step(*args, 1)
    with pytest.raises((TypeError, ValueError)):
        T.adamw_step(p, g, m, v, 1, units=([], []))
    with pytest.raises(ValueError):
        T.adamw_state(p, 16)
    assert all(torch.equal(x, y) for x, y in zip(kept, p + m + v))
    # the same gradient for two parameters is only read
    q = [torch.zeros(300, device="cuda") for _ in range(2)]
    mm, vv, _ = T.adamw_state(q)
    T.adamw_step(q, [g[0], g[0]], mm, vv, 1)
    assert torch.equal(q[0], q[1]) and q[0].any()
    T.adamw_step([], [], [], [], 1)


# ---- without a GPU ----------------------------------------------------------------------------
def test_argument_errors_without_a_gpu():
    L, E_ARG, E_RANGE = T.lib(), -1, -2

    def call(n=1, tensor={}, **change):
        a = T._Adamw(32, 1, None, 1e-3, 0.9, 0.999, 1e-8, 0.01, None, None, 0)
        for name, x in change.items():
            setattr(a, name, x)
        t = (T._AdamwTensor * 2)()
        for i in range(2):
            t[i] = T._AdamwTensor(0, 0, 10, 0x1000 * (4 * i + 1), 0x1000 * (4 * i + 2), 0x1000 * (4 * i + 3), 0x1000 * (4 * i + 4), 0x100, 0x200)
        for name, x in tensor.items():
            setattr(t[0], name, x)
        return L.taser_adamw_step(ctypes.byref(a), t, n, None)

    assert L.taser_adamw_step(None, None, 0, None) == E_ARG and call(n=-1) == E_ARG and call(n=2 ** 31) == E_RANGE and call(n=0) == 0
    for change in (dict(bits=16), dict(beta1=1.0), dict(beta2=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(weight_decay=-0.5), dict(lr=-1.0), dict(lr=float("inf")), dict(step=0)):
        assert call(**change) == E_ARG, change
    for tensor, code in ((dict(elements=-1), E_ARG), (dict(type=3), E_ARG), (dict(grad_type=-1), E_ARG), (dict(elements=2 ** 35 + 1), E_RANGE), (dict(param=None), E_ARG), (dict(m=None), E_ARG),
                         (dict(v=None), E_ARG), (dict(m=0x1000), E_ARG), (dict(v=0x1000 + 39), E_ARG), (dict(grad=0x1000 + 20), E_ARG)):
        assert call(tensor=tensor) == code, tensor
    assert call(bits=8, tensor=dict(m_unit=None)) == E_ARG and call(bits=8, tensor=dict(v_unit=0x100)) == E_ARG
    assert call(n=2, tensor=dict(param=0x5000)) == E_ARG and "overlap" in T.last_error()
    assert call(tensor=dict(elements=0)) == 0 and call(tensor=dict(grad=None)) == 0
    moments = lambda m=16, v=16, n=5, kind=0, out=16: L.taser_adamw_moments(m, v, 16, 16, n, kind, out, out, None)
    assert moments(m=None) == moments(v=None) == moments(n=-1) == moments(kind=3) == moments(out=None) == E_ARG and moments(n=2 ** 36) == E_RANGE and moments(n=0, m=None) == 0


@pytest.mark.parametrize("name, size", [("step_at", 8), ("lr_at", 4), ("grad_scale", 4)])
def test_numbers_that_lie_in_what_is_written_are_refused(name, size):
    """Found without a GPU: the call is refused before anything is launched."""
    starts, units = (0x1000, 0x3000, 0x4000), (0x100, 0x200)   # of 10 elements' parameters, m and v; of a unit each
    for bits in (32, 8):
        ends = (40, 40 if bits == 32 else 10, 40 if bits == 32 else 10) + (4, 4)
        for at, length in list(zip(starts + units, ends))[:3 if bits == 32 else 5]:
            for place in (at, at + length - 1, at - size + 1):
                a = T._Adamw(bits, 1, None, 1e-3, 0.9, 0.999, 1e-8, 0.01, None, None, 0)
                setattr(a, name, place)
                t = (T._AdamwTensor * 1)(T._AdamwTensor(0, 0, 10, 0x1000, 0x2000, 0x3000, 0x4000, 0x100, 0x200))
                assert T.lib().taser_adamw_step(ctypes.byref(a), t, 1, None) == -1 and "that is written" in T.last_error(), (bits, hex(place))


def test_the_oracle_against_another_form_of_the_step():
    rng = np.random.default_rng(1)
    p, g = rng.standard_normal(50), rng.standard_normal((6, 50))
    q = torch.nn.Parameter(torch.from_numpy(p.copy()))
    optimizer = torch.optim.AdamW([q], lr=0.03, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.2)
    m = v = np.zeros(50)
    for i in range(6):
        q.grad = torch.from_numpy(g[i])
        optimizer.step()
        got, _ = O.adamw(p, g[i], m, v, "float32", i + 1, 0.03, 0.8, 0.95, 1e-6, 0.2)
        p, m, v = got["p"], got["m"], got["v"]
    assert np.abs(p - q.detach().numpy()).max() < 1e-12


def test_the_oracle_rounds_without_bias():
    """Codes by evenly spread chances: a value's mean comes to itself, within a half of the chances' spacing."""
    rng = np.random.default_rng(2)
    for quad in (False, True):
        x = np.append(rng.random(20) ** 3, 1.0)
        power, most = (4, 255.0) if quad else (2, 127.0)
        chances = (np.arange(1024) + 0.5) / 1024
        codes = np.stack([O.adamw_codes(x, np.full(21, u), quad)[0] for u in chances])
        values = (codes / most) ** power
        spacing = ((codes.min(0) + 1.0) / most) ** power - (codes.min(0) / most) ** power
        assert (np.abs(values.mean(0) - x) <= spacing / 1024 + 1e-12).all() and codes[:, -1].min() == most


def test_the_oracles_random_words(golden_dir):
    """Published answers of Philox4x32-10."""
    rows = [line.split() for line in open(os.path.join(golden_dir, "philox4x32_10_kat.txt")) if line.strip() and not line.startswith("#")]
    assert len(rows) >= 3
    for row in rows:
        numbers = [int(x, 16) for x in row[-10:]]
        got = O.philox([np.array([x]) for x in numbers[:4]], numbers[4:6])
        assert [int(x[0]) for x in got] == numbers[6:]


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-16, 1e-12])
def test_small_gradients_beside_a_small_eps(bits, eps):
    """Second moments below 2^-126 count where eps does not outweigh them. The first step, from moments of zero: m / sqrt(v) is 0.1 / sqrt(0.001) of the gradient's sign. In 32
    bits (1 - beta2) g^2 is off by 2^-24 of itself twice and by half the spacing of the smallest numbers, 2^-150, of either product; its root has half of that."""
    g = torch.Generator().manual_seed(12)
    for size in (1e-18, 1e-19, 3e-17, 1e-15, 1e-3):
        grad = ((0.5 + torch.rand(700, generator=g)) * (1 - 2.0 * torch.randint(0, 2, (700,), generator=g)) * size).cuda()
        p = [torch.zeros(700, device="cuda")]
        m, v, units = T.adamw_state(p, bits)
        T.adamw_step(p, [grad], m, v, 1, lr=0.01, eps=eps, weight_decay=0.0, units=units)
        x, e = _arr(grad), float(np.float32(eps))
        root = np.abs(x)   # of v / c2
        off = root * ((2 * O.E32 * 0.001 * x * x + 2.0 ** -150 * 1.001) / (0.001 * x * x) + 6 * O.E32)
        want = -0.01 * x / (root + e)
        far = np.abs(_arr(p[0]) - want) - np.abs(want) * (off / (root + e - off) + 12 * O.E32)
        assert (far <= 0).all(), (size, float(far.max()), float(want[0]), p[0][0].item())


@gpu
def test_small_gradients_for_some_steps_in_8_bits():
    """Equal gradients of 1e-18 or 1e-16 and an eps of 0: m / sqrt(v) is theirs' sign at each step, so that a parameter moves by lr. Every moment is its block's
    largest, kept as its unit: three roundings a step of m, of v's root no more, and v's own of 2^-149 of some 1e-39 at first."""
    for size in (1e-18, 1e-16):
        p = [torch.zeros(600, device="cuda")]
        m, v, units = T.adamw_state(p, 8)
        for step in range(1, 6):
            T.adamw_step(p, [torch.full((600,), size, device="cuda")], m, v, step, lr=0.01, eps=0.0, weight_decay=0.0, units=units)
        assert (p[0].double() + 0.05).abs().max() <= 0.05 * (5 * 12 * O.E32 + 5 * 2.0 ** -149 / 1e-39), size


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-40, 2.0 ** -149, 1e-38, 1e-37])
def test_an_eps_at_the_end_of_the_numbers(bits, eps):
    """Elements without a gradient so far stay as they are (0 / eps), the others move by lr."""
    p = [torch.ones(300, device="cuda")]
    grad = torch.zeros(300, device="cuda")
    grad[::3] = 0.5
    m, v, units = T.adamw_state(p, bits)
    for step in (1, 2):
        T.adamw_step(p, [grad], m, v, step, lr=0.01, eps=eps, weight_decay=0.0, units=units)
    assert (p[0][1::3] == 1).all() and (p[0][2::3] == 1).all()
    assert (p[0][::3] - 0.98).abs().max() <= 0.02 * 24 * O.E32 + 4 * O.E32


@gpu
def test_a_step_past_64_bits_is_refused(monkeypatch):
    for native in (True, False):
        with monkeypatch.context() as change:
            if not native:
                change.setattr(T, "_native", Absent())
            p, g = [torch.zeros(5, device="cuda")], [torch.ones(5, device="cuda")]
            m, v, _ = T.adamw_state(p)
            for step in (2 ** 63, 2 ** 64 + 1, -2 ** 64 + 1, -2 ** 63 - 1):
                with pytest.raises(ValueError):
                    T.adamw_step(p, g, m, v, step)
            assert not p[0].any() and not m[0].any()
            T.adamw_step(p, g, m, v, 2 ** 63 - 1)
            assert p[0].all()
