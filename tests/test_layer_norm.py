"""Layer norm and its gradient against their definition in 64 bits (GPU), the oracle's gradient against differences (CPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2402_05396_amd as T
from oracle import operators as O

KINDS = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
gpu = pytest.mark.gpu


class Absent:
    def __getattr__(self, name):
        return lambda *a: None


def _case(kind, R, W, kept=None, weight=True, bias=True, seed=0, offset=0.3, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g)
    to = KINDS[kept or kind]
    return dict(kind=kind, kept=kept or kind, x=(offset + spread * rnd(R, W)).to(KINDS[kind]), dout=rnd(R, W).to(KINDS[kind]), weight=(1 + 0.3 * rnd(W)).to(to) if weight else None,
                bias=(0.3 * rnd(W)).to(to) if bias else None)


def _run(c, eps=1e-5, stream=None):
    d = lambda t: None if t is None else t.cuda()
    x, dout, weight, bias = (d(c[n]) for n in ("x", "dout", "weight", "bias"))
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    out, stats = T.layer_norm(x, weight, bias, eps=eps, want_stats=True, stream=stream)
    if stream is None:
        again = T.layer_norm(x, weight, bias, eps=eps)
        assert torch.equal(torch.isnan(again), torch.isnan(out)) and torch.equal(torch.nan_to_num(again), torch.nan_to_num(out))
    got = (out, *T.layer_norm_grad(dout, x, stats, weight, bias, stream=stream))
    if stream is not None:
        stream.synchronize()
    return dict(zip(("out", "dx", "dweight", "dbias"), got), stats=stats)


def _check(c, eps=1e-5):
    arr = lambda t: None if t is None else t.double().numpy()
    got = _run(c, eps)
    eps32 = float(np.float32(eps))
    want, off = O.layer_norm(arr(c["x"]), c["kind"], arr(c["weight"]), arr(c["bias"]), eps32, arr(c["dout"]), c["kept"])
    for n in ("out", "dx", "dweight", "dbias"):
        if n[1:] in ("weight", "bias") and c[n[1:]] is None:
            assert got[n] is None
            continue
        assert got[n].dtype == KINDS[c["kept"] if n[1:] in ("weight", "bias") else c["kind"]]
        x = got[n].double().cpu().numpy()
        far = np.abs(x - want[n]) - off[n]
        assert x.shape == want[n].shape and (far <= 0).all(), (n, float(far.max()))
    return got


WIDTHS = [1, 2, 3, 7, 8, 9, 31, 33, 64, 65, 100, 127, 129, 256, 257, 511, 513, 1000, 1023, 1025, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 20_001, 40_000]


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("W", WIDTHS)
def test_against_64_bits(kind, W):
    for i, R in enumerate((1, 5, 67)):
        _check(_case(kind, R, W, kept=None if i != 1 else "float32", weight=i != 2, bias=i != 2 or W % 2 == 0, seed=W + R))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [(20_000, 5), (12_000, 100), (9000, 300), (3001, 1023), (2500, 2048), (1100, 5000), (700, 9000), (300, 17_000)])
def test_many_rows(kind, shape):
    """More rows than there are groups of threads: each goes through several."""
    _check(_case(kind, *shape, seed=shape[1]))


@gpu
def test_weight_or_bias_alone():
    for W in (60, 3000, 20_000):
        for weight, bias in ((True, False), (False, True), (False, False)):
            for kept in ("bfloat16", "float32"):
                _check(_case("bfloat16", 21, W, kept=kept, weight=weight, bias=bias, seed=W))


@gpu
@pytest.mark.parametrize("W", [50, 1000, 30_000])
def test_rows_far_from_zero(W):
    """What is away from the mean keeps its digits: a difference of sums of squares would have none left."""
    _check(_case("float32", 40, W, offset=3000.0, seed=1))
    for kind in ("float16", "bfloat16"):
        _check(_case(kind, 40, W, offset=30.0, spread=4.0, seed=2))


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_rows_of_one_value(kind):
    for W in (1, 100, 5000, 20_000):
        c = _case(kind, 6, W, seed=3)
        c["x"][:] = torch.arange(6, dtype=torch.float32)[:, None].to(KINDS[kind])
        got = _run(c)
        # the mean of W equal numbers is off by (W + 4) 2^-24 of them at most, and what is left is multiplied by 1 / sqrt(eps)
        most = (W + 4) * O.E32 * 5 * 1e-5 ** -0.5 * 3
        assert (got["out"].double().cpu() - c["bias"].double()).abs().max() <= most + O.U[kind] * 2, W


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_a_row_that_is_not_finite_stays_by_itself(kind):
    for W in (20, 1000, 5000, 20_000):
        c = _case(kind, 300, W, seed=4)
        clean = _run(c)
        c["x"][7, W // 2], c["x"][9, 0], c["dout"][11, 3] = float("nan"), float("inf"), float("nan")
        got = _run(c)
        rows = torch.ones(300, dtype=torch.bool)
        rows[[7, 9]] = False
        assert torch.equal(got["out"][rows], clean["out"][rows]) and torch.isnan(got["out"][~rows]).any(1).all()
        rows[11] = False
        assert torch.equal(got["dx"][rows], clean["dx"][rows]) and torch.isnan(got["dx"][~rows]).any(1).all()
        assert torch.isnan(got["dweight"]).any() and torch.isnan(got["dbias"][3]) and torch.isfinite(got["dbias"][4:]).all()


@gpu
def test_strides_alignment_streams_and_bits(monkeypatch):
    for kind, R, W in (("bfloat16", 333, 100), ("float16", 40, 1023), ("float32", 70, 777), ("bfloat16", 65, 5001), ("float32", 9, 20_000)):
        c = _case(kind, R, W, seed=5)
        want = _run(c)
        side = torch.cuda.Stream()
        wide = dict(c)
        for name in ("x", "dout"):
            t = torch.full((R, W + 7), float("nan"), dtype=KINDS[kind]).cuda()
            t[:, 3:W + 3] = c[name].cuda()
            wide[name] = t[:, 3:W + 3]
        wide["x"], wide["dout"] = (type("Given", (), {"cuda": lambda self, t=wide[n]: t})() for n in ("x", "dout"))   # as it is, strides and all
        for given in (c, wide):
            for stream in (None, side):
                got = _run(given, stream=stream)
                assert all(torch.equal(got[n], want[n]) for n in want), (kind, W)
        with monkeypatch.context() as m:
            m.setattr(T, "_native", Absent())
            got = _run(c)
            assert all(torch.equal(got[n], want[n]) for n in want)


@gpu
def test_graph():
    for W in (100, 3000, 17_000):
        c = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in _case("bfloat16", 50, W, kept="float32", seed=6).items()}

        def call():
            out, stats = T.layer_norm(c["x"], c["weight"], c["bias"], want_stats=True)
            return (out, *T.layer_norm_grad(c["dout"], c["x"], stats, c["weight"], c["bias"]))
        call()
        graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        with torch.cuda.graph(other, pool=graph.pool()):
            again = call()
        for _ in range(3):
            c["x"].normal_()
            graph.replay()
            other.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) and torch.equal(e, b) for a, b, e in zip(got, call(), again))


@gpu
def test_without_rows():
    x, w = torch.zeros((0, 9), device="cuda"), torch.ones(9, device="cuda")
    out, stats = T.layer_norm(x, w, w, want_stats=True)
    dx, dw, db = T.layer_norm_grad(x, x, stats, w, w)
    assert out.shape == dx.shape == (0, 9) and stats.shape == (0, 2) and not dw.any() and not db.any()


@gpu
def test_gradient_against_differences():
    """(f(x + h e) - f(x - h e)) / 2h of sum(out * dout) along a unit direction: out's roundings, 16 * 2^-24 of each product's size, over the step, and
    the third derivative, at most some 60 |dout| / deviation^3 for a row, times h^2 / 6."""
    for W in (20, 300, 6000):
        c = _case("float32", 10, W, seed=7)
        got = _run(c)
        h, g = 2.0 ** -6, torch.Generator().manual_seed(8)
        for name, of in (("x", "dx"), ("weight", "dweight"), ("bias", "dbias")):
            e = torch.randn(c[name].shape, generator=g)
            e /= e.norm()
            f = lambda t: (_run(dict(c, **{name: t}))["out"].double().cpu() * c["dout"].double()).sum()
            up, down = c[name] + h * e, c[name] - h * e
            step = (up.double() - down.double()) / (2 * h)
            slope, want = float(f(up) - f(down)) / (2 * h), float((got[of].double().cpu() * step).sum())
            noise = 16 * O.E32 * float((got["out"].double().cpu().abs() * c["dout"].double().abs()).sum()) / h
            third = 60 * float(c["dout"].double().norm()) * h * h / 6 if name == "x" else 0.0
            assert abs(slope - want) <= noise + third, (W, name, slope, want)


@gpu
def test_refusals_of_the_binding():
    x, w = torch.zeros((4, 9), device="cuda"), torch.zeros(9, device="cuda")
    out, stats = T.layer_norm(x, w, w, want_stats=True)
    T.layer_norm_grad(x, x, stats, w, w)
    for bad in ((x.double(), w, w), (x[0], w, w), (x.t(), None, None), (x.cpu(), w, w), (x, w.half(), w.half()), (x, w.double(), None), (x, torch.zeros(18, device="cuda")[::2], w), (x, w.cpu(), w),
                (x.half(), w, w.half())):
        with pytest.raises(TypeError):
            T.layer_norm(*bad)
    for bad in ((x, w[:8], w), (x, w, w[None])):
        with pytest.raises(ValueError):
            T.layer_norm(*bad)
    for eps in (-1e-5, float("nan"), float("inf")):
        with pytest.raises(T.TaserError):
            T.layer_norm(x, w, w, eps=eps)
    for bad in ((x.half(), x, stats, w, w), (x, x, stats.double(), w, w), (x.t(), x.t(), stats, None, None)):
        with pytest.raises(TypeError):
            T.layer_norm_grad(*bad)
    for bad in ((x[:3], x, stats, w, w), (x, x, stats[:3], w, w)):
        with pytest.raises(ValueError):
            T.layer_norm_grad(*bad)
    assert T.layer_norm_grad_bytes(x, w, w) > 0


# ---- without a GPU ----------------------------------------------------------------------------
def test_argument_errors_without_a_gpu():
    L, one, E_ARG, E_RANGE = T.lib(), ctypes.c_void_p(16), -1, -2

    def block(**change):
        n = T._Norm(0, 0, 3, 5, 5, 16, 16, 16, 1e-5)
        for name, x in change.items():
            setattr(n, name, x)
        return ctypes.byref(n)

    size = ctypes.c_uint64()
    assert L.taser_layer_norm(None, one, one, None) == E_ARG and L.taser_layer_norm_grad_bytes(None, ctypes.byref(size)) == E_ARG
    for change, code in ((dict(type=3), E_ARG), (dict(weight_type=1), E_ARG), (dict(rows=-1), E_ARG), (dict(width=0), E_ARG), (dict(width=2 ** 26 + 2 ** 8, x_stride=2 ** 27), E_RANGE),
                         (dict(rows=2 ** 32), E_RANGE), (dict(rows=2 ** 23, width=20_000, x_stride=20_000), E_RANGE), (dict(eps=-1.0), E_ARG), (dict(eps=float("nan")), E_ARG),
                         (dict(x=None), E_ARG), (dict(x_stride=4), E_ARG)):
        assert L.taser_layer_norm(block(**change), one, one, None) == code, change
        assert L.taser_layer_norm_grad(block(**change), one, one, 2 ** 27, one, one, one, one, 2 ** 60, None) == code, change
    assert L.taser_layer_norm(block(), None, one, None) == E_ARG and L.taser_layer_norm_grad_bytes(block(), None) == E_ARG
    assert L.taser_layer_norm_grad_bytes(block(), ctypes.byref(size)) == 0 and size.value > 0
    grad = lambda stats=one, dout=one, stride=5, dx=one, dw=one, work=one, n=2 ** 40: L.taser_layer_norm_grad(block(), stats, dout, stride, dx, dw, one, work, n, None)
    assert grad(stats=None) == grad(dout=None) == grad(stride=4) == grad(dx=None) == grad(work=None) == grad(n=size.value - 1) == grad(work=ctypes.c_void_p(8)) == E_ARG
    assert L.taser_layer_norm(block(rows=0), None, None, None) == 0 and L.taser_layer_norm_grad(block(rows=0), None, None, 5, None, None, None, None, 0, None) == 0


def test_the_oracle_against_differences():
    c = _case("float32", 3, 6, seed=9)
    x, dout, w, b = (c[n].double().numpy() for n in ("x", "dout", "weight", "bias"))
    want, h = O.layer_norm(x, "float32", w, b, 1e-5, dout)[0], 2.0 ** -16
    for name, at, of in (("dx", x, 0), ("dweight", w, 1), ("dbias", b, 2)):
        for i in np.ndindex(at.shape):
            f = []
            for sign in (1, -1):
                args = [x.copy(), w.copy(), b.copy()]
                args[of][i] += sign * h
                f.append((O.layer_norm(args[0], "float32", args[1], args[2], 1e-5)[0]["out"] * dout).sum())
            assert abs((f[0] - f[1]) / (2 * h) - want[name][i]) < 1e-6, (name, i)
