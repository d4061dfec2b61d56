"""The bias by distance as a tensor and its table's gradient, against their definitions (GPU), and their refusals."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2402_05396_amd as T
from oracle import operators as O

KINDS = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
gpu = pytest.mark.gpu


def _case(kind, B, H, Lq, Lk, n, seed, positions="near", shared=False):
    g = torch.Generator().manual_seed(seed)
    P = 1 if shared else B
    if positions == "near":
        qp, kp = torch.arange(Lq)[None].repeat(P, 1) + torch.randint(-3, 9, (P, 1), generator=g), torch.arange(Lk)[None].repeat(P, 1)
        bounds = torch.arange(n - 1) * 2 - n
    elif positions == "any":
        qp, kp = torch.randint(-99, 99, (P, Lq), generator=g), torch.randint(-99, 99, (P, Lk), generator=g)
        bounds = torch.sort(torch.randint(-150, 150, (n - 1,), generator=g)).values   # some twice: buckets that nothing falls into
    else:
        far = 2 ** 61
        qp, kp = torch.randint(-far, far, (P, Lq), generator=g), torch.randint(-far, far, (P, Lk), generator=g)
        bounds = torch.sort(torch.randint(-far, far, (n - 1,), generator=g)).values
    table = torch.randn((H, n), generator=g).to(KINDS[kind])
    dbias = torch.randn((B, H, Lq, Lk), generator=g).to(KINDS[kind])
    bucket = np.stack([O.buckets(bounds.tolist(), qp[b % P].tolist(), kp[b % P].tolist()) for b in range(B)])
    return table, dbias, bounds, qp, kp, bucket


SIZES = [(1, 1, 1, 1, 1), (1, 3, 5, 7, 2), (2, 12, 33, 129, 32), (3, 2, 1, 513, 64), (1, 16, 130, 64, 17), (2, 1, 64, 1000, 9), (1, 130, 3, 70, 64), (4, 5, 200, 8, 3)]


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("positions", ["near", "any", "far"])
def test_bias_and_gradient(kind, size, positions):
    B, H, Lq, Lk, n = size
    for shared in (False, True) if B == 1 else (False,):
        table, dbias, bounds, qp, kp, bucket = _case(kind, B, H, Lq, Lk, n, B + H + Lq, positions, shared)
        dev = [t.cuda() for t in (bounds, qp, kp)]
        got = T.relative_bias(table.cuda(), *dev).cpu()
        want = table[:, torch.from_numpy(bucket)].transpose(0, 1)
        assert got.dtype == table.dtype and torch.equal(got, want)   # values are moved, not computed
        dtable = T.relative_bias_grad(dbias.cuda(), *dev)
        assert dtable.shape == table.shape and dtable.dtype == dbias.dtype
        x = dbias.double().numpy()
        for i in range(n):
            here = (bucket == i)[:, None]
            sums, mags = (x * here).sum((0, 2, 3)), (np.abs(x) * here).sum((0, 2, 3))
            # N values are added in 32 bits in chains of at most N, then rounded to the type
            off = (here.sum() * O.E32) * mags
            off = off + O.U[kind] * (np.abs(sums) + off) + O.TINY[kind]
            assert (np.abs(dtable[:, i].double().cpu().numpy() - sums) <= off).all(), i


@gpu
def test_strides_of_the_gradient():
    table, dbias, bounds, qp, kp, _ = _case("bfloat16", 2, 6, 40, 77, 9, 1)
    dev = [t.cuda() for t in (bounds, qp, kp)]
    want = T.relative_bias_grad(dbias.cuda(), *dev)
    wide = torch.full((2, 40, 6, 80), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = wide[..., 1:78].transpose(1, 2)
    view.copy_(dbias)
    assert torch.equal(T.relative_bias_grad(view, *dev), want)
    shared = dbias[:1].cuda().expand(2, -1, -1, -1)
    assert torch.equal(T.relative_bias_grad(shared, *dev), T.relative_bias_grad(shared.contiguous(), *dev))
    for _ in range(3):
        assert torch.equal(T.relative_bias_grad(dbias.cuda(), *dev), want)


@gpu
def test_equal_to_the_bias_in_attention():
    """Attention with q = 0 has the softmax of the bias as weights; its table gradient is the bias gradient of dx."""
    table, _, bounds, qp, kp, bucket = _case("float32", 2, 3, 9, 50, 12, 4)
    dev = [t.cuda() for t in (bounds, qp, kp)]
    v = torch.randn((2, 50, 3, 16), device="cuda")
    out = T.cross_attention(torch.zeros((2, 9, 3, 16), device="cuda"), v, v, bias=(table.cuda(), *dev))
    w = torch.softmax(T.relative_bias(table.cuda(), *dev).double(), 3)
    want = torch.matmul(w, v.double().transpose(1, 2)).transpose(1, 2)
    assert (out.double() - want).abs().max() < 64 * 2.0 ** -24 * v.abs().max()


@gpu
def test_sizes_of_zero_streams_and_halves(monkeypatch):
    class Absent:
        def __getattr__(self, name):
            return lambda *a: None
    table, dbias, bounds, qp, kp, _ = _case("float16", 2, 3, 20, 30, 5, 2)
    dev = [t.cuda() for t in (bounds, qp, kp)]
    for B, Lq, Lk in ((0, 2, 3), (2, 0, 3), (2, 3, 0)):
        p = [torch.zeros((max(B, 1) if not B else B, n), dtype=torch.int64, device="cuda")[:B] for n in (Lq, Lk)]
        assert T.relative_bias(table.cuda(), dev[0], *p).numel() == 0
        d = T.relative_bias_grad(torch.ones((B, 3, Lq, Lk), device="cuda", dtype=torch.float16), dev[0], *p)
        assert d.shape == (3, 5) and not d.any()
    a, b = T.relative_bias(table.cuda(), *dev), T.relative_bias_grad(dbias.cuda(), *dev)
    side = torch.cuda.Stream()
    x = dbias.cuda()
    side.wait_stream(torch.cuda.current_stream())
    c, d = T.relative_bias(table.cuda(), *dev, stream=side), T.relative_bias_grad(x, *dev, stream=side)
    side.synchronize()
    assert torch.equal(a, c) and torch.equal(b, d)
    monkeypatch.setattr(T, "_native", Absent())
    assert torch.equal(T.relative_bias(table.cuda(), *dev), a) and torch.equal(T.relative_bias_grad(dbias.cuda(), *dev), b)
    assert T.relative_bias_bytes(dbias.cuda(), *dev) > 0


@gpu
def test_refusals_of_the_binding():
    table, dbias, bounds, qp, kp, _ = _case("float16", 2, 3, 20, 30, 5, 2)
    t, x, b, q, k = (a.cuda() for a in (table, dbias, bounds, qp, kp))
    for bad in ((t.double(), b, q, k), (t.t(), b, q, k), (t, b.int(), q, k), (t, b, q[0], k), (t, b, q.int(), k), (t, b, q, k.cpu())):
        with pytest.raises(TypeError):
            T.relative_bias(*bad)
    for bad in ((t, b[:2], q, k), (t[:, :4].contiguous(), b, q, k), (t, b, q, torch.cat([k, k[:1]]))):
        with pytest.raises(ValueError):
            T.relative_bias(*bad)
    for bad in ((x.double(), b, q, k), (x[0], b, q, k), (x.transpose(2, 3), b, q, k)):
        with pytest.raises(TypeError):
            T.relative_bias_grad(*bad)
    for bad in ((x[:1], b, q, k), (x[:, :, :5], b, q, k), (x, b, q, k[:, :7].contiguous())):
        with pytest.raises(ValueError):
            T.relative_bias_grad(*bad)
    with pytest.raises(T.TaserError):
        T.relative_bias(torch.zeros((3, 65), device="cuda"), torch.zeros(64, dtype=torch.int64, device="cuda"), q, k)


def test_argument_errors_without_a_gpu():
    L, one, E_ARG, E_RANGE = T.lib(), ctypes.c_void_p(16), -1, -2
    size = ctypes.c_uint64()
    strides = (ctypes.c_int64 * 3)(60, 20, 5)

    def block(**change):
        d = T._Distances(0, 3, 4, 2, 4, 5, 16, 16, 16, 0, 0)
        for n, x in change.items():
            setattr(d, n, x)
        return ctypes.byref(d)

    assert L.taser_relative_bias_bytes(block(), ctypes.byref(size)) == 0 and size.value > 0
    for change, code in ((dict(type=7), E_ARG), (dict(heads=0), E_ARG), (dict(heads=70000), E_RANGE), (dict(buckets=0), E_RANGE), (dict(buckets=65), E_RANGE), (dict(batch=-1), E_ARG),
                         (dict(keys=-1), E_ARG), (dict(keys=2 ** 31), E_RANGE), (dict(queries=2 ** 31), E_RANGE), (dict(batch=2 ** 20, queries=2 ** 20), E_RANGE), (dict(bounds=None), E_ARG),
                         (dict(query_pos=None), E_ARG), (dict(key_pos=None), E_ARG)):
        assert L.taser_relative_bias_bytes(block(**change), ctypes.byref(size)) == code, change
        assert L.taser_relative_bias(block(**change), one, one, None) == code, change
        assert L.taser_relative_bias_grad(block(**change), one, strides, one, one, 1 << 40, None) == code, change
    assert L.taser_relative_bias_bytes(None, None) == E_ARG
    assert L.taser_relative_bias(block(), None, one, None) == E_ARG
    assert L.taser_relative_bias(block(), one, None, None) == E_ARG
    assert L.taser_relative_bias_grad(block(), None, strides, one, one, 1 << 40, None) == E_ARG
    assert L.taser_relative_bias_grad(block(), one, None, one, one, 1 << 40, None) == E_ARG
    assert L.taser_relative_bias_grad(block(), one, strides, None, one, 1 << 40, None) == E_ARG
    assert L.taser_relative_bias_grad(block(), one, strides, one, None, 1 << 40, None) == E_ARG
    assert L.taser_relative_bias_grad(block(), one, strides, one, ctypes.c_void_p(8), 1 << 40, None) == E_ARG
    assert L.taser_relative_bias_grad(block(), one, strides, one, one, 8, None) == E_RANGE


def test_calls_that_no_launch_can_take_are_refused():
    """Fewer than 2^32 threads to a launch: 64 for each 256 states of a query (512 in 16 bits)."""
    one = ctypes.c_void_p(16)
    for batch, queries, keys in ((2 ** 26, 1, 1), (2 ** 15, 2 ** 11, 25), (2 ** 28, 16, 1), (1, 2 ** 25, 300)):
        d = T._Distances(0, 3, 4, batch, queries, keys, 16, 16, 16, 0, 0)
        assert T.lib().taser_relative_bias(ctypes.byref(d), one, one, None) == -2 and "launch" in T.last_error(), T.last_error()
