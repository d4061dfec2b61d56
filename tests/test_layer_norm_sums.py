"""Layer norm's sums over rows and columns: no element is left out or taken twice. The bounds count the additions that a number goes through in
the kernels, not all numbers of a sum, and the inputs have large elements where a loop could stop early (GPU); that such a loss would be
past the bounds is shown with the results of one (CPU)."""
import numpy as np
import pytest
import torch

import paper_2402_05396_amd as T
from oracle import operators as O
from test_layer_norm import KINDS, _case, _run

gpu = pytest.mark.gpu
EPS32 = float(np.float32(1e-5))
# The last of a row in its first piece, in a part of a wave, in the last of its waves; rows that are held by a block, and past what it holds.
WIDTHS = [1, 5, 8, 9, 17, 33, 100, 129, 257, 513, 1023, 1025, 2049, 4097, 8192, 8193, 16_384, 16_385, 20_001, 32_768, 32_769, 40_000, 65_537]


def depth(R, W):
    """Additions that a number goes through at most: in a row's sums up to 32 columns of a thread (past 32768 columns W / 1024 and a piece's 8), 6 across a
    wave and 16 waves; in the sums over rows R / 256 of a group, 3 across a wave, 8 groups, 16 parts and 5 across them."""
    return 64 + W // 1024, 48 + R // 256


def _arr(t):
    return None if t is None else t.double().cpu().numpy()


def _expected(c):
    return O.layer_norm(_arr(c["x"]), c["kind"], _arr(c["weight"]), _arr(c["bias"]), EPS32, _arr(c["dout"]), c["kept"], depth(*c["x"].shape))


def _compare(c, want, off):
    got = _run(c)
    got.update(mean=got["stats"][:, :1], rstd=got["stats"][:, 1:])
    for n in want:
        far = np.abs(_arr(got[n]) - want[n]) - off[n]
        assert (far <= 0).all(), (n, float(far.max()))


def _marked(kind, R, W, seed):
    """A large element at the end of each row and of each column."""
    c = _case(kind, R, W, kept="float32", seed=seed)
    c["x"][:, -1], c["dout"][:, -1] = 12.0, 12.0
    c["dout"][-1] = 4.0
    return c


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("W", WIDTHS)
def test_whole_rows(kind, W):
    for R in (1, 7):
        c = _marked(kind, R, W, seed=W)
        _compare(c, *_expected(c))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [(70_000, 1), (70_001, 5), (70_000, 30), (40_001, 64), (40_000, 100), (20_001, 200), (10_001, 300), (10_000, 500), (4001, 1023), (1500, 5000), (700, 9000)])
def test_all_rows(kind, shape):
    """More rows than twice the groups of threads that there are (32768 of 8 lanes, 16384 of 16, and so on to one row a block): each goes through three."""
    c = _marked(kind, *shape, seed=shape[1])
    _compare(c, *_expected(c))
    # sums of whole numbers are exact
    c["dout"] = torch.randint(-3, 4, shape, generator=torch.Generator().manual_seed(0)).to(KINDS[kind])
    assert np.array_equal(_arr(_run(c)["dbias"]), _arr(c["dout"]).sum(0))
    # gradients of a few rows alone: what is left of the sums are a few numbers
    few = [0, shape[0] // 2 - 1, shape[0] - 2, shape[0] - 1]
    c["dout"] = torch.zeros_like(c["dout"])
    c["dout"][few] = 1.0
    xhat = O.layer_norm(_arr(c["x"][few]), kind, eps=EPS32, kept="float32")[0]["out"]
    ex = O.layer_norm(_arr(c["x"][few]), "float32", eps=EPS32, depth=depth(*shape))[1]["out"]
    got = _run(c)
    assert (np.abs(_arr(got["dweight"]) - xhat.sum(0)) <= ex.sum(0) + 12 * O.E32 * np.abs(xhat).sum(0)).all()
    assert (got["dbias"] == 4.0).all()


@gpu
@pytest.mark.parametrize("W", [50, 1000, 8193, 30_000, 40_000])
def test_rows_far_from_zero(W):
    """What is away from the mean keeps its digits, also in long rows."""
    c = _case("float32", 20, W, offset=3000.0, seed=1)
    _compare(c, *_expected(c))


@gpu
@pytest.mark.parametrize("W", [1, 100, 5000, 20_000, 40_000])
def test_rows_of_one_value(W):
    c = _case("float32", 6, W, seed=3)
    c["x"][:] = torch.arange(6, dtype=torch.float32)[:, None]
    _compare(c, *_expected(c))


# ---- without a GPU ----------------------------------------------------------------------------
def _past(lossy, want, off, names):
    """Whether results of a loss are past the bounds, each of them."""
    return all((np.abs(lossy[n] - want[n]) > off[n]).any() for n in names)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("W", [w for w in WIDTHS if w > 1])
def test_a_lost_column_is_past_the_bounds(kind, W):
    """The last column left out of the mean, of the variance, or of either sum of the gradient."""
    c = _marked(kind, 2, W, seed=W)
    want, off = _expected(c)
    x, w, b, dout = (_arr(c[n]) for n in ("x", "weight", "bias", "dout"))

    def results(mean, var, g_sums):
        rstd = 1 / np.sqrt(var + EPS32)
        xhat, g = (x - mean) * rstd, dout * w
        s, t = (y[:, :g_sums].sum(1, keepdims=True) / W for y in (g, g * xhat))
        return dict(out=xhat * w + b, mean=mean, rstd=rstd, dx=rstd * (g - s - xhat * t))

    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    assert not _past(results(mean, var, W), want, off, ["out"]) and not _past(results(mean, var, W), want, off, ["dx"])
    less = x[:, :-1].sum(1, keepdims=True) / W
    assert _past(results(less, ((x - less) ** 2).mean(1, keepdims=True), W), want, off, ["mean"])
    assert _past(results(mean, ((x - mean)[:, :-1] ** 2).sum(1, keepdims=True) / W, W), want, off, ["rstd"])
    if kind == "float32" or W < 10_000:   # (a wider row's dx in 16 bits is rounded to more than its share of the sums)
        assert _past(results(mean, var, W - 1), want, off, ["dx"])


@pytest.mark.parametrize("shape", [(70_001, 5), (40_000, 100), (10_000, 500)])
def test_a_lost_row_is_past_the_bounds(shape):
    c = _marked("float32", *shape, seed=shape[1])
    want, off = _expected(c)
    less = {"dweight": want["dweight"] - _arr(c["dout"])[-1] * (_arr(c["x"])[-1] - want["mean"][-1]) * want["rstd"][-1], "dbias": want["dbias"] - _arr(c["dout"])[-1]}
    assert _past(less, want, off, ["dweight", "dbias"])


@pytest.mark.parametrize("W", [1000, 30_000])
def test_other_forms_of_the_variance_are_past_the_bounds(W):
    """Of rows far from zero: sums of squares less the mean's, in 32 bits; and nothing at all."""
    c = _case("float32", 20, W, offset=3000.0, seed=1)
    want, off = _expected(c)
    x = c["x"].numpy()
    var = (x * x).mean(1, keepdims=True, dtype=np.float32) - x.mean(1, keepdims=True, dtype=np.float32) ** 2
    assert _past({"rstd": 1 / np.sqrt(np.maximum(var, 0) + np.float32(1e-5))}, want, off, ["rstd"])
    assert _past({n: np.zeros_like(y) for n, y in want.items()}, want, off, ["out", "mean", "rstd", "dx", "dweight", "dbias"])
