"""Training with an adaptive sampler, whole steps of it: candidates found, ten of them chosen by the sampler's logits, the chosen
neighbors' rows attended to by their roots with a bias by how long ago each interaction was, and both models updated: the
aggregation by its loss, the sampler by the clipped policy loss of what it chose (TASER, arXiv 2402.05396, Alg. 1, with one layer of
aggregation).

The graph and its task are synthetic: one edge in five says something about its later roots' labels, and the sampler sees in the
edge's row which ones do. A uniform choice therefore keeps a fifth of such edges where a root has many candidates; the share kept
is printed beside the loss.

    python -m paper_2402_05396_amd.adaptive_training [--steps 60] [--roots 4096] [--type bfloat16]
"""
import argparse
import json

import torch

import paper_2402_05396_amd as T


class CrossAttention(torch.autograd.Function):
    """cross_attention with its gradient, a table of biases by distance included. (A gradient of the gradient is an error.)"""

    @staticmethod
    def forward(ctx, q, k, v, table, bounds, query_pos, key_pos, lengths):
        out, stats = T.cross_attention(q, k, v, lengths=lengths, bias=(table, bounds, query_pos, key_pos), want_stats=True)
        ctx.save_for_backward(q, k, v, table, bounds, query_pos, key_pos, lengths, out, stats)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, table, bounds, query_pos, key_pos, lengths, out, stats = ctx.saved_tensors
        dq, dk, dv, dtable = T.cross_attention_grad(dout.contiguous(), q, k, v, out, stats, lengths=lengths, bias=(table, bounds, query_pos, key_pos))
        return dq, dk, dv, dtable, None, None, None, None


class PolicyLoss(torch.autograd.Function):
    """The sum of policy_loss over rows and picks; its gradient comes with the forward pass. (Its gradient is an error.)"""

    @staticmethod
    def forward(ctx, logits, actions, advantage, old_logp, count):
        loss, _, grad = T.policy_loss(logits, actions, advantage, old_logp=old_logp, count=count)
        ctx.save_for_backward(grad)
        return loss.sum()

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        return ctx.saved_tensors[0] * dloss, None, None, None, None


def synthetic(nodes, edges, dim, seed, device):
    """A graph with time-sorted edges, their rows (element 0: whether the edge says something, 1: what), and per edge the same."""
    rng = torch.Generator().manual_seed(seed)
    src, dst = (torch.randint(0, nodes, (edges,), generator=rng, dtype=torch.int32) for _ in range(2))
    ts = torch.sort(torch.randint(0, 1000 * edges, (edges,), generator=rng)).values
    table = 0.5 * torch.randn((edges, dim), generator=rng)
    tells = torch.rand(edges, generator=rng) < 0.2
    says = torch.randint(0, 2, (edges,), generator=rng) * 2 - 1
    table[:, 0] = tells.float()
    table[:, 1] = says.float()
    eid = torch.arange(edges, dtype=torch.int32)
    graph = T.tcsr_build(*(t.to(device) for t in (torch.cat([src, dst]), torch.cat([dst, src]), torch.cat([ts, ts]), torch.cat([eid, eid]))), nodes)
    return graph, table.to(device), int(ts[-1]) + 1


class Trainer:
    """Both models of the example and what they train on."""

    def __init__(self, roots=4096, candidates=25, picks=10, heads=2, head_dim=32, dim=32, nodes=2000, edges=100_000, dtype=torch.bfloat16, seed=0):
        device = torch.device("cuda")
        self.graph, self.table, self.end = synthetic(nodes, edges, dim, seed, device)
        self.roots, self.candidates, self.picks, self.heads, self.head_dim, self.nodes = roots, candidates, picks, heads, head_dim, nodes
        self.dtype, self.rng = dtype, torch.Generator().manual_seed(seed + 1)
        width = heads * head_dim

        def weights(*shape):
            return (0.3 * torch.randn(shape, generator=self.rng)).to(device).requires_grad_()

        self.query, self.key, self.value, self.answer = weights(width), weights(dim, width), weights(dim, width), weights(width)
        self.score = torch.zeros(dim + 1, device=device, requires_grad=True)   # the sampler: a candidate's row and how often its node comes
        # Powers of two apart: recent interactions are told apart finely, old ones coarsely.
        self.bounds = 2 ** torch.arange(12, 12 + 15, device=device, dtype=torch.int64)
        self.bias = torch.zeros((heads, 16), device=device, requires_grad=True)
        self.model = torch.optim.Adam([self.query, self.key, self.value, self.answer, self.bias], lr=0.02)
        self.sampler = torch.optim.Adam([self.score], lr=0.1)

    def aggregate(self, rows, times, kept):
        """[R, width]: what each root's kept neighbors' rows come to."""
        r, n = kept["nbr"].shape
        q = self.query.to(self.dtype).view(1, 1, self.heads, -1).expand(r, 1, self.heads, self.head_dim)
        k, v = ((rows @ w).to(self.dtype).view(r, n, self.heads, self.head_dim) for w in (self.key, self.value))
        out = CrossAttention.apply(q, k, v, self.bias.to(self.dtype), self.bounds, times.view(r, 1), kept["ts"], kept["count"])
        return out.reshape(r, -1).float()

    def step(self, number):
        """One step of both models -> {loss, share of the kept neighbors that say something}."""
        roots = torch.randint(0, self.nodes, (self.roots,), generator=self.rng, dtype=torch.int32).cuda()
        times = torch.randint(self.end // 2, self.end, (self.roots,), generator=self.rng).cuda()
        found = T.sample_temporal(self.graph, roots, times, self.candidates, 1, T.RECENT, number)[0]
        count, dim = found["count"], self.table.shape[1]
        freq, _ = T.candidate_encodings(found["nbr"], count, want_identity=False)
        rows = T.gather_features(self.table, found["eid"].reshape(-1)).view(self.roots, self.candidates, dim)
        tells = rows[..., 0] * (found["eid"] >= 0)
        label = ((tells * rows[..., 1]).sum(1) > 0).float()

        seen = torch.cat([rows, freq.unsqueeze(-1).float()], -1)
        logits = seen @ self.score
        there = torch.arange(self.candidates, device="cuda") < count.unsqueeze(1)
        chances = torch.where(there, logits.detach(), -torch.inf).softmax(1).nan_to_num()
        weight = (chances * 65535).to(torch.int32) + 1
        actions, _, kept = T.select_weighted(weight, count, self.picks, number, 0, candidates=found)
        nothing = torch.zeros(actions.shape, device="cuda")
        _, old_logp, _ = T.policy_loss(logits.detach(), actions, nothing, count=count, want_grad=False)

        chosen = T.gather_features(self.table, kept["eid"].reshape(-1)).view(self.roots, self.picks, dim)
        losses = torch.nn.functional.binary_cross_entropy_with_logits(self.aggregate(chosen, times, kept) @ self.answer, label, reduction="none")
        self.model.zero_grad()
        losses.mean().backward()
        self.model.step()

        reward = -losses.detach()
        advantage = ((reward - reward.mean()) / (reward.std() + 1e-6)).unsqueeze(1).expand_as(actions).contiguous()
        for _ in range(4):   # steps away from where the choice was made: that is what the clipped ratio is for
            self.sampler.zero_grad()
            (PolicyLoss.apply(seen @ self.score, actions, advantage, old_logp, count) / actions.numel()).backward()
            self.sampler.step()
        kept_rows = kept["eid"] >= 0
        return {"loss": losses.mean().item(), "share": ((chosen[..., 0] * kept_rows).sum() / kept_rows.sum()).item()}


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--roots", type=int, default=4096)
    ap.add_argument("--type", choices=["float32", "float16", "bfloat16"], default="bfloat16")
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args(argv)
    trainer = Trainer(roots=args.roots, dtype=getattr(torch, args.type), seed=args.seed)
    steps = [trainer.step(i) for i in range(args.steps)]
    for i in range(0, args.steps, max(1, args.steps // 10)):
        print("step %d: loss %.4f, kept %.3f" % (i, steps[i]["loss"], steps[i]["share"]), flush=True)
    result = {"steps": args.steps, "first": steps[0], "last": steps[-1]}
    print(json.dumps(result))
    return steps


if __name__ == "__main__":
    main()
