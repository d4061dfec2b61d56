"""Layer norm, draws, the policy loss and the AdamW step together, as a policy's training step has them; and their use by the example."""
import numpy as np
import pytest
import torch

import paper_2402_05396_amd as T
from oracle import operators as O

pytestmark = pytest.mark.gpu
LR, KL = 0.05, 0.1


class Policy:
    """Logits are the norm of a state, scaled and shifted candidate by candidate: weight and bias are what is learned."""

    def __init__(self, rows, width, picks, bits, kind=torch.float32, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.state = torch.randn((rows, width), generator=g).to(kind).cuda()
        self.uniform = torch.rand((rows, picks), generator=g).cuda()
        self.gain = torch.randn((rows, picks), generator=g).cuda()
        self.ref = (-3 + torch.randn((rows, picks), generator=g)).cuda()
        self.params = [(1 + 0.2 * torch.randn(width, generator=g)).cuda(), (0.3 * torch.randn(width, generator=g)).cuda()]
        self.m, self.v, self.units = T.adamw_state(self.params, bits)
        self.step_number = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(self):
        self.step_number.add_(1)
        logits, stats = T.layer_norm(self.state, *self.params, want_stats=True)
        actions, old = T.policy_draw(logits, self.uniform, temperature=0.9, top_k=20, top_p=0.9)
        loss, logp, dlogits = T.policy_loss(logits, actions, self.gain, old_logp=old, ref_logp=self.ref, kl=KL)
        _, dweight, dbias = T.layer_norm_grad(dlogits, self.state, stats, *self.params)
        T.adamw_step(self.params, [dweight, dbias], self.m, self.v, self.step_number, lr=LR, units=self.units, weight_decay=0.0)
        return logits, actions, old, loss, dlogits, dweight, dbias

    def copy(self):
        other = object.__new__(Policy)
        clone = lambda x: x.clone() if isinstance(x, torch.Tensor) else None if x is None else type(x)(clone(y) for y in x)
        other.__dict__ = {n: clone(x) for n, x in self.__dict__.items()}
        return other


@pytest.mark.parametrize("width", [50, 700])
def test_a_step_against_64_bits(width):
    rows, picks = 30, 3
    p = Policy(rows, width, picks, 32)
    before = [x.double().cpu().numpy() for x in p.params]
    logits, actions, old, loss, dlogits, dweight, dbias = (x.cpu() for x in p.step())
    arr = lambda t: t.double().cpu().numpy()
    x, eps = arr(p.state), float(np.float32(1e-5))
    want, off = O.layer_norm(x, "float32", *before, eps)
    assert (np.abs(arr(logits) - want["out"]) <= off["out"]).all()
    got = arr(logits)   # each operator from here on against its definition, at what it was given
    drawn, l, eoff, sure = O.policy_draw(got, arr(p.uniform), temperature=np.float32(0.9), top_k=20, top_p=np.float32(0.9))
    assert sure.mean() > 0.95 and ((actions.numpy() == drawn) | ~sure).all()
    want, off = O.policy_loss(got, actions.numpy(), arr(p.gain), "float32", arr(old), arr(p.ref), kl=KL)
    assert (np.abs(arr(loss) - want["loss"]) <= off["loss"]).all() and (np.abs(arr(dlogits) - want["grad"]) <= off["grad"]).all()
    want, off = O.layer_norm(x, "float32", *before, eps, arr(dlogits))
    for name, g in (("dweight", dweight), ("dbias", dbias)):
        assert (np.abs(arr(g) - want[name]) <= off[name]).all(), name
    for now, was, g in zip(p.params, before, (dweight, dbias)):
        want, off = O.adamw(was, arr(g), np.zeros(width), np.zeros(width), "float32", 1, lr=LR, decay=0.0)
        assert (np.abs(arr(now) - want["p"]) <= off["p"]).all()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("rows,width,kind", [(300, 25, torch.float32), (40, 3001, torch.bfloat16), (3, 40_000, torch.float16)])
def test_steps_replayed_from_a_graph(bits, rows, width, kind):
    """The whole step is launches of kernels: captured, it goes on as it does eagerly, with the program's own work between."""
    p = Policy(rows, width, 2, bits, kind)
    q = p.copy()
    p.copy().step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = p.step()
    for i in range(4):
        for x in (p, q):
            g = torch.Generator("cuda").manual_seed(i)
            x.uniform.uniform_(generator=g)
            x.state.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        want = q.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all(torch.equal(a, b) for n in ("params", "m", "v") for a, b in zip(getattr(p, n), getattr(q, n))), i


def test_two_streams_at_once():
    """Steps of two policies on two streams: workspaces are each call's own."""
    policies = [Policy(20, 20_000, 2, 32, seed=i) for i in range(2)]
    want = [p.copy() for p in policies]
    for _ in range(3):
        for p in want:
            p.step()
    streams = [torch.cuda.Stream() for _ in policies]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for p, s in zip(policies, streams):
            with torch.cuda.stream(s):
                p.step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for p, q in zip(policies, want) for a, b in zip(p.params + p.m, q.params + q.m))


def test_layer_norm_as_a_function():
    from paper_2402_05396_amd.adaptive_training import LayerNorm
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((37, 64), generator=g, device="cuda").requires_grad_()
    weight, bias = (torch.randn(64, generator=g, device="cuda").requires_grad_() for _ in range(2))
    dout = torch.randn((64, 37), generator=g, device="cuda").t()
    got = torch.autograd.grad(LayerNorm.apply(x, weight, bias, 1e-5), (x, weight, bias), dout)
    arr = lambda t: t.detach().double().cpu().numpy()
    want, off = O.layer_norm(arr(x), "float32", arr(weight), arr(bias), float(np.float32(1e-5)), arr(dout))
    for name, y in zip(("dx", "dweight", "dbias"), got):
        assert (np.abs(arr(y) - want[name]) <= off[name]).all(), name
    out = LayerNorm.apply(x, weight, bias, 1e-5)
    (dx,) = torch.autograd.grad((out * out).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (dx * x).sum().backward()


@pytest.mark.parametrize("options", [["--norm"], ["--bits", "8"], ["--norm", "--bits", "8", "--type", "float32"]])
def test_the_example_runs(options):
    from paper_2402_05396_amd import adaptive_training
    steps = adaptive_training.main(["--steps", "3", "--roots", "512"] + options)
    assert len(steps) == 3 and all(np.isfinite(s["loss"]) for s in steps)
