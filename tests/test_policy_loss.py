"""The clipped policy loss and its gradient against their definition in 64 bits (GPU), the oracle's gradient against differences (CPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2402_05396_amd as T
from oracle import operators as O

KINDS = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
gpu = pytest.mark.gpu


def _case(kind, R, W, n, seed=0, old=True, ref=True, count=False, weight=True, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g)
    c = dict(kind=kind, logits=(rnd(R, W) * spread).to(KINDS[kind]), actions=torch.randint(-1, W, (R, n), generator=g, dtype=torch.int32), advantage=rnd(R, n), old=None, ref=None, count=None,
             weight=None)
    if n > 1:
        c["actions"][:, 1] = c["actions"][:, 0]   # the same action twice
    lp = torch.gather(torch.log_softmax(c["logits"].float(), 1), 1, c["actions"].clamp(min=0).long())
    if old:
        c["old"] = lp + 0.3 * rnd(R, n)
    if ref:
        c["ref"] = lp + 0.3 * rnd(R, n)
    if count:
        c["count"] = torch.randint(0, W + 2, (R,), generator=g, dtype=torch.int32)
    if weight:
        c["weight"] = torch.rand((R, n), generator=g) * (torch.rand((R, n), generator=g) < 0.8)
    return c


def _run(c, **more):
    d = lambda t: None if t is None else t.cuda()
    return T.policy_loss(d(c["logits"]), d(c["actions"]), d(c["advantage"]), d(c["old"]), d(c["ref"]), count=d(c["count"]), weight=d(c["weight"]), clip_low=0.2, clip_high=0.3, kl=0.1, **more)


def _check(c):
    arr = lambda t: None if t is None else t.double().numpy()
    got = dict(zip(("loss", "logp", "grad"), _run(c)))
    want, off = O.policy_loss(arr(c["logits"]), c["actions"].numpy(), arr(c["advantage"]), c["kind"], arr(c["old"]), arr(c["ref"]), c["count"], arr(c["weight"]), 0.2, 0.3, 0.1)
    for n, x in got.items():
        x = x.double().cpu().numpy()
        far = np.abs(x - want[n]) - off[n]
        assert x.shape == want[n].shape and (far <= 0).all(), (n, float(far.max()))
    return got


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [(1, 1, 1), (700, 25, 10), (333, 16, 4), (65, 17, 3), (64, 33, 1), (40, 64, 64), (50, 3, 60), (33, 65, 1), (9, 1000, 5), (7, 4096, 1), (5, 4099, 64), (3, 70_001, 2),
                                   (2, 140_000, 1)])
def test_against_64_bits(kind, shape):
    for old, ref, count, weight in ((True, True, False, True), (True, False, True, False), (False, False, True, True), (False, True, False, False)):
        _check(_case(kind, *shape, seed=shape[1], old=old, ref=ref, count=count, weight=weight))


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_what_takes_no_part_is_not_read(kind):
    for R, W, n in ((50, 25, 6), (6, 300, 6), (4, 9000, 3)):
        c = _case(kind, R, W, n, seed=4, count=True)
        c["count"][0], c["count"][1] = 0, 1
        past = torch.arange(W)[None] >= c["count"][:, None]
        c["logits"] = torch.where(past, torch.tensor(float("nan"), dtype=KINDS[kind]), c["logits"])
        c["old"] = torch.nan_to_num(c["old"], nan=-1.0)
        c["ref"] = torch.nan_to_num(c["ref"], nan=-1.0)
        none = c["weight"] == 0
        for name in ("old", "ref", "advantage"):
            c[name] = torch.where(none, torch.tensor(float("nan")), c[name])   # nor what is given for an action of weight 0
        clean = dict(c, logits=torch.where(past, torch.zeros((), dtype=KINDS[kind]), c["logits"]))
        for name in ("old", "ref", "advantage"):
            clean[name] = torch.where(none, torch.zeros(()), c[name])
        got = _run(c)
        for a, b in zip(got, _check(clean).values()):
            assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_logits_of_minus_infinity(kind):
    """Candidates that a model has ruled out have no weight; an action among them has a log-probability of minus infinity."""
    for R, W in ((20, 30), (5, 500), (3, 7000)):
        c = _case(kind, R, W, 2, seed=9, ref=False)
        c["logits"][:, ::3] = -float("inf")
        c["actions"][:] = torch.tensor([1, 4], dtype=torch.int32)
        c["old"] = torch.randn((R, 2)) - 3
        _check(c)
        c["actions"][0, 0] = 3
        loss, logp, grad = _run(c)
        assert logp[0, 0] == -float("inf") and torch.isfinite(loss).all() and torch.isfinite(grad).all() and not grad[:, ::3].any()


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_large_logits(kind):
    for W in (20, 200, 5000):
        _check(_case(kind, 6, W, 3, seed=2, spread=300.0, old=False, ref=False))


@gpu
def test_strides_alignment_streams_and_bits():
    for kind, R, W, n in (("bfloat16", 9, 25, 3), ("float16", 5, 4097, 3), ("float32", 4, 777, 1), ("bfloat16", 3, 66_000, 1)):
        c = _case(kind, R, W, n, seed=1, count=True)
        want = _run(c)
        wide = torch.full((R, W + 7), float("nan"), dtype=KINDS[kind])
        wide[:, 3:W + 3] = c["logits"]
        d = lambda t: t.cuda()
        args = [d(wide)[:, 3:W + 3], d(c["actions"]), d(c["advantage"]), d(c["old"]), d(c["ref"])]
        more = dict(count=d(c["count"]), weight=d(c["weight"]), clip_low=0.2, clip_high=0.3, kl=0.1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for stream in (None, side):
            got = T.policy_loss(*args, stream=stream, **more)
            side.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b)
        loss, logp, none = T.policy_loss(*args, want_grad=False, **more)
        assert none is None and torch.equal(loss, want[0]) and torch.equal(logp, want[1])


@gpu
def test_gradient_against_differences():
    """(f(x + h e) - f(x - h e)) / 2h of the summed losses in single precision: the losses' roundings, 2^-24 * 8 of the sum of their
    magnitudes, over a step of 2^-5, and the third derivative along a unit direction, at most the first's order, times h^2 / 6."""
    for W, n in ((25, 5), (300, 2), (6000, 1)):
        c = _case("float32", 40, W, n, seed=3, weight=False)
        loss, _, grad = _run(c)
        # advantages of both signs: away from the ends of the clip the loss is smooth
        e = torch.randn(c["logits"].shape, generator=torch.Generator().manual_seed(1))
        e /= e.norm()
        h = 2.0 ** -5
        f = lambda x: _run(dict(c, logits=x))[0].double()
        up, down = f(c["logits"] + h * e), f(c["logits"] - h * e)
        slope, want = float((up - down).sum()) / (2 * h), float((grad.double().cpu() * e.double()).sum())
        noise = 8 * 2.0 ** -24 * float(loss.double().abs().sum()) / h
        # an action whose ratio crosses an end of the clip within the step: its slope may count for all or nothing
        lp, ends = [_run(dict(c, logits=x))[1].cpu() for x in (c["logits"] + h * e, c["logits"] - h * e)], []
        for bound in (0.8, 1.3):
            r = [torch.exp(x - c["old"]) - bound for x in lp]
            ends.append(float(((r[0] * r[1] <= 0) & (c["actions"] >= 0)).float().mul(c["advantage"].abs() * 2).sum()) * float(max((x - y).abs().max() for x, y in [lp])) / (2 * h))
        assert abs(slope - want) <= noise + sum(ends) + h * h / 6 * 8 * float(grad.double().norm()), (W, slope, want)


@gpu
def test_graph_and_halves(monkeypatch):
    class Absent:
        def __getattr__(self, name):
            return lambda *a: None
    for W in (25, 5000):
        c = _case("float32", 30, W, 3, seed=5)
        want = _run(c)
        logits = c["logits"].cuda()
        args = [c[n].cuda() for n in ("actions", "advantage", "old", "ref")]
        call = lambda: T.policy_loss(logits, *args, weight=wt, clip_low=0.2, clip_high=0.3, kl=0.1)
        wt = c["weight"].cuda()
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for _ in range(3):
            logits.normal_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, call()))
        with monkeypatch.context() as m:
            m.setattr(T, "_native", Absent())
            assert all(torch.equal(a, b) for a, b in zip(_run(c), want))
    empty = T.policy_loss(torch.zeros((0, 5), device="cuda"), torch.zeros((0, 2), dtype=torch.int32, device="cuda"), torch.zeros((0, 2), device="cuda"))
    assert [x.shape for x in empty] == [(0, 2), (0, 2), (0, 5)]


@gpu
def test_with_the_sampler_that_chooses():
    """select_weighted's choices are the actions, its candidates' counts the rows' lengths."""
    R, m, k = 500, 25, 10
    g = torch.Generator("cuda").manual_seed(0)
    logits = torch.randn((R, m), device="cuda", generator=g)
    count = torch.randint(0, m + 1, (R,), device="cuda", generator=g, dtype=torch.int32)
    weight = (torch.softmax(logits, 1) * 2 ** 30).clamp(min=1).int()
    sel, kept, _ = T.select_weighted(weight, count, k, 1, 0)
    loss, logp, grad = T.policy_loss(logits, sel, torch.ones((R, k), device="cuda"), count=count)
    taken = (sel >= 0)
    assert torch.equal(taken.sum(1).int(), kept)
    assert torch.equal(loss, torch.where(taken, -1.0, 0.0)) and (logp[taken] < 1e-6).all() and not logp[~taken].any()
    assert grad.sum(1).abs().max() < 1e-5 and not grad[torch.arange(m, device="cuda")[None] >= count[:, None]].any()


@gpu
def test_refusals_of_the_binding():
    x, a, v = torch.zeros((4, 9), device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    T.policy_loss(x, a, v)
    for bad in ((x.double(), a, v), (x[0], a, v), (x.t(), a, v), (x.cpu(), a, v), (x, a.long(), v), (x, a, v.half()), (x, a, v, v.double()), (x, a, v, None, v.t())):
        with pytest.raises(TypeError):
            T.policy_loss(*bad)
    with pytest.raises(TypeError):
        T.policy_loss(x, a, v, count=torch.zeros(4, device="cuda"))
    for bad in ((x[:3], a, v), (x, a, v[:3]), (x, a, v, v[:, :1].contiguous())):
        with pytest.raises(ValueError):
            T.policy_loss(*bad)
    with pytest.raises(ValueError):
        T.policy_loss(x, a, v, count=torch.zeros(3, dtype=torch.int32, device="cuda"))
    for bad in (dict(clip_low=-0.1), dict(clip_high=-0.1), dict(kl=-1.0), dict(kl=float("nan"))):
        with pytest.raises(T.TaserError):
            T.policy_loss(x, a, v, **bad)
    with pytest.raises(T.TaserError):
        T.policy_loss(x, torch.zeros((4, 65), dtype=torch.int32, device="cuda"), torch.zeros((4, 65), device="cuda"))


# ---- without a GPU ----------------------------------------------------------------------------
def test_argument_errors_without_a_gpu():
    L, one, E_ARG, E_RANGE = T.lib(), ctypes.c_void_p(16), -1, -2

    def block(**change):
        p = T._PolicyBatch(0, 2, 3, 5, 5, 16, None, 16, 16, None, None, None, 0.2, 0.2, 0.0)
        for n, x in change.items():
            setattr(p, n, x)
        return ctypes.byref(p)

    assert L.taser_policy_loss(None, one, one, one, None) == E_ARG
    for change, code in ((dict(type=3), E_ARG), (dict(rows=-1), E_ARG), (dict(width=0), E_ARG), (dict(picks=0), E_ARG), (dict(picks=65), E_RANGE), (dict(width=2 ** 31), E_RANGE),
                         (dict(rows=2 ** 31), E_RANGE), (dict(clip_low=-1.0), E_ARG), (dict(kl=float("nan")), E_ARG), (dict(logits=None), E_ARG), (dict(actions=None), E_ARG),
                         (dict(advantage=None), E_ARG), (dict(logits_stride=4), E_ARG)):
        assert L.taser_policy_loss(block(**change), one, one, one, None) == code, change
    assert L.taser_policy_loss(block(), None, one, one, None) == E_ARG
    assert L.taser_policy_loss(block(), one, None, one, None) == E_ARG
    assert L.taser_policy_loss(block(rows=0), None, None, None, None) == 0


def test_the_oracle_against_differences():
    for old, ref in ((True, True), (True, False)):
        c = _case("float32", 6, 7, 3, seed=8, old=old, ref=ref, count=True)
        arr = lambda t: None if t is None else t.double().numpy()
        run = lambda x: O.policy_loss(x, c["actions"].numpy(), arr(c["advantage"]), "float32", arr(c["old"]), arr(c["ref"]), c["count"], arr(c["weight"]), 0.2, 0.3, 0.1)[0]
        x = arr(c["logits"])
        grad, h = run(x)["grad"], 2.0 ** -16
        for i in np.ndindex(x.shape):
            up, down = x.copy(), x.copy()
            up[i] += h
            down[i] -= h
            assert abs((run(up)["loss"].sum() - run(down)["loss"].sum()) / (2 * h) - grad[i]) < 1e-7, i


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_rows_without_an_action_that_counts_have_no_gradient(kind):
    """Padded rows: no action, or actions of weight 0, over logits that are NaN, infinite or ruled out."""
    for W in (20, 64, 300, 5000, 70_000):
        x = torch.zeros((6, W), dtype=KINDS[kind])
        x[0], x[1], x[2] = float("nan"), -float("inf"), float("inf")
        x[3, W // 2] = x[5, W // 2] = float("nan")
        a = torch.full((6, 3), -1, dtype=torch.int32)
        a[3:, 1] = 2
        weight = torch.ones((6, 3))
        weight[3] = 0.0
        loss, logp, grad = T.policy_loss(x.cuda(), a.cuda(), torch.ones((6, 3)).cuda(), weight=weight.cuda())
        assert not grad[:4].any() and not loss[:4].any() and not logp[:3].any(), W
        assert abs(float(grad[4, 2]) + 1 - 1 / W) < 2.0 ** -8 and float(grad[4].float().sum().abs()) < 2.0 ** -8, W


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_nan_among_logits_of_minus_infinity(kind):
    """A NaN whose neighbors are all ruled out reaches the row's results, wherever in the row it lies."""
    for W in (20, 300, 5000, 70_000):
        for at in (3, 11, W // 2, W - 2):
            x = torch.full((3, W), -float("inf"), dtype=KINDS[kind])
            x[:, 1] = 0.5
            x[1, at] = float("nan")
            x[2, W - 1] = 0.5
            a = torch.ones((3, 1), dtype=torch.int32)
            loss, logp, grad = T.policy_loss(x.cuda(), a.cuda(), torch.ones((3, 1)).cuda())
            assert torch.isnan(logp[1]).all() and torch.isnan(grad[1, 1]) and torch.isfinite(logp[[0, 2]]).all() and torch.isfinite(grad[[0, 2]]).all(), (W, at)


def test_calls_that_no_launch_can_take_are_refused():
    """Fewer than 2^32 threads to a launch: 16 to 64 a short row, a block of 256 or 1024 a longer one."""
    one = ctypes.c_void_p(16)
    for rows, width, picks in ((2 ** 28, 5, 2), (2 ** 26, 5, 40), (2 ** 24, 100, 2), (2 ** 22, 10_000, 2)):
        p = T._PolicyBatch(0, picks, rows, width, width, 16, None, 16, 16, None, None, None, 0.2, 0.2, 0.0)
        assert T.lib().taser_policy_loss(ctypes.byref(p), one, one, one, None) == -2 and "launch" in T.last_error(), T.last_error()


@gpu
@pytest.mark.parametrize("W", [25, 300, 5000])
def test_kl_term_of_a_policy_close_to_its_reference(W):
    """exp(t) - t - 1 at the t that the kernel has (the returned log-probability's difference, exact where they are close): at most 16
    roundings off. The gradient's slope, 1 - exp(t), likewise, beside those of W terms in the softmax."""
    def term(t):   # its series, 20 terms of it, and the function itself past 1/2
        s = np.zeros_like(t)
        for n in range(22, 1, -1):
            s = (s * t + 1) / n
        return np.where(np.abs(t) < 0.5, t * t * s, np.expm1(t) - t)

    for apart in (3.0, 0.7, 0.4, 0.1, 1e-2, 1e-3, 3e-4, 1e-4, 1e-6):
        g = torch.Generator().manual_seed(W)
        x = torch.randn((200, W), generator=g).cuda()
        a = torch.randint(0, W, (200, 1), generator=g, dtype=torch.int32).cuda()
        none = torch.zeros((200, 1), device="cuda")
        _, logp, _ = T.policy_loss(x, a, none)
        ref = logp + apart * torch.randn((200, 1), generator=g).cuda()
        loss, again, grad = T.policy_loss(x, a, none, ref_logp=ref, kl=0.5)
        assert torch.equal(again, logp)
        t = (ref - logp).double().cpu().numpy()
        want, got = 0.5 * term(t), loss.double().cpu().numpy()
        assert (got >= 0).all() and (np.abs(got - want) <= 16 * O.E32 * want + O.END32).all(), (apart, float(np.abs(got / want - 1).max()))
        slope, chance = -0.5 * np.expm1(t), np.exp(logp.double().cpu().numpy())
        at = grad.double().cpu().numpy()[np.arange(200), a.cpu().numpy()[:, 0]][:, None]
        assert (np.abs(at - slope * (1 - chance)) <= (W + 40) * O.E32 * np.abs(slope)).all(), apart
