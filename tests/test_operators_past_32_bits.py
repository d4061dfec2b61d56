"""Rows and tensors whose elements are more than 32 bits count: the last of them are what a call of their own gives."""
import pytest
import torch

import paper_2402_05396_amd as T

pytestmark = pytest.mark.gpu
MORE = 2 ** 32


@pytest.fixture(autouse=True)
def memory_of_its_own():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _filled(*shape, scale=1.0):
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator("cuda").manual_seed(0)
    for part in t.view(-1).split(2 ** 28):
        part.normal_(generator=g)
    return t.mul_(scale) if scale != 1.0 else t


def test_layer_norm():
    W = 8192
    R = MORE // W + 300
    x = _filled(R, W)
    weight, bias = torch.randn(W, device="cuda"), torch.randn(W, device="cuda")
    out, stats = T.layer_norm(x, weight, bias, want_stats=True)
    few, s = T.layer_norm(x[-200:].clone(), weight, bias, want_stats=True)
    assert torch.equal(out[-200:], few) and torch.equal(stats[-200:], s)
    dx, dweight, dbias = T.layer_norm_grad(out, x, stats, weight, bias)
    assert torch.equal(dx[-200:], T.layer_norm_grad(few, x[-200:].clone(), s, weight, bias)[0])
    # sums of R numbers in 32 bits, of magnitudes that are their own sum of magnitudes at most
    want, size = sum(p.double().sum(0) for p in out.split(2 ** 14)), sum(p.double().abs().sum(0) for p in out.split(2 ** 14))
    assert ((dbias.double() - want).abs() <= (R + 8) * 2.0 ** -24 * size).all()


def test_draws():
    W = 100_001
    R = MORE // W + 50
    x = _filled(R, W, scale=2.0)
    u = torch.rand((R, 2), device="cuda")
    for settings in (dict(top_p=0.9), dict(top_k=40), {}):
        actions, logp = T.policy_draw(x, u, **settings)
        few, l = T.policy_draw(x[-40:].clone(), u[-40:].clone(), **settings)
        assert torch.equal(actions[-40:], few) and (logp[-40:] - l).abs().max() <= 2 * (W + 80) * 2.0 ** -24


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    n, tail = MORE + 3000, 2000   # the tail begins with a block of 256
    tail += (n - tail) % 256
    p, g = _filled(n), _filled(n, scale=0.01)
    m, v, units = T.adamw_state([p], bits)
    q = [p[-tail:].clone()]
    other = T.adamw_state(q, bits)
    for step in (1, 2):
        T.adamw_step([p], [g], m, v, step, lr=0.1, units=units)
        T.adamw_step(q, [g[-tail:].clone()], other[0], other[1], step, lr=0.1, units=other[2])
        if bits == 32 or step == 1:   # (codes go by an element's place: what follows from them differs)
            assert torch.equal(p[-tail:], q[0])
    if bits == 32:
        assert torch.equal(m[0][-tail:], other[0][0]) and torch.equal(v[0][-tail:], other[1][0])
    else:
        a = T.adamw_moments(m[0], v[0], (units[0][0], units[1][0]), dtype=torch.bfloat16)
        b = T.adamw_moments(m[0][-tail:].clone(), v[0][-tail:].clone(), tuple(u[0][-(-(-tail // 256)):].clone() for u in units), dtype=torch.bfloat16)
        assert all(torch.equal(x[-tail:], y) for x, y in zip(a, b)) and a[1][-tail:].all()


def test_layer_norms_sums_over_the_last_rows():
    """Only rows past the border have a gradient: dbias is their sum of whole numbers, exactly, and dweight a sum of 300 products that are off by
    four roundings each (what is away from the mean, its reciprocal deviation, the product, the sum so far)."""
    W, few = 8192, 300
    R = MORE // W + few
    x = _filled(R, W)
    weight, bias = torch.randn(W, device="cuda"), torch.randn(W, device="cuda")
    out, stats = T.layer_norm(x, weight, bias, want_stats=True)
    del out
    dout = torch.zeros((R, W), dtype=torch.bfloat16, device="cuda")
    dout[-few:] = torch.randint(-3, 4, (few, W), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    dx, dweight, dbias = T.layer_norm_grad(dout, x, stats, weight, bias)
    assert not dx[:-few].any() and dx[-few:].any(1).all()
    tail = dout[-few:].double()
    assert torch.equal(dbias.double(), tail.sum(0))
    each = tail * (x[-few:].double() - stats[-few:, :1].double()) * stats[-few:, 1:].double()
    assert ((dweight.double() - each.sum(0)).abs() <= (few + 4) * 2.0 ** -24 * each.abs().sum(0)).all()
    lost = (each[0].abs() > (few + 4) * 2.0 ** -24 * each.abs().sum(0)).float().mean()   # of one row: seen wherever its gradient is not 0
    assert lost > 0.8
