"""A worker's training step on the library's own operators, and rounds of it through the server path (Algorithm 4: compute
the gradient, send it, receive the mean, update).

The model is the smallest one that meets all of them: token embedding, dropout, one causal attention block with a residual
dropout, and an output layer tied to the embedding table.  Plain matrix products are torch's; embedding, dropout, attention
and their gradients are the library's.  The gradient is written straight into one flat buffer in the order of the plan's
tensors, which is what dblp_packetize reads.

    python -m paper_2605_01989_b200.worker          # four workers, 2 % of the packets lost, a few rounds
"""
import math

import torch

from . import binding as dblp
from . import workloads as wl

EMBED_SITE, RESIDUAL_SITE = 0, 1          # which dropout of a step a mask belongs to


class TokenModel:
    """Parameters in fp32 in one flat vector, in the order of `numel`: table, qkv projection, output projection."""

    def __init__(self, rows, heads, head_dim, device, seed=0):
        self.rows, self.heads, self.head_dim, self.width = rows, heads, head_dim, heads * head_dim
        d = self.width
        self.shapes = [(rows, d), (d, 3 * d), (d, d)]
        self.numel = [a * b for a, b in self.shapes]
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.flat = torch.randn(sum(self.numel), generator=g, device=device) * 0.02
        self.table, self.w_qkv, self.w_out = self.views(self.flat)

    def views(self, flat):
        """The tensors of a flat vector laid out like the parameters."""
        return [v.view(s) for v, s in zip(flat.split(self.numel), self.shapes)]


class Worker:
    """One worker: buffers for a batch of `batch` sequences of `tokens` tokens, and its flat fp32 gradient."""

    def __init__(self, model, batch, tokens, p=0.1, seed=0):
        self.model, self.p, self.seed = model, p, seed
        dev, d, n = model.flat.device, model.width, batch * tokens
        half = dict(dtype=torch.bfloat16, device=dev)
        heads = (batch, tokens, model.heads, model.head_dim)
        self.grad = torch.zeros(sum(model.numel), device=dev)
        self.emb, self.x0, self.x1, self.dx = (torch.empty((n, d), **half) for _ in range(4))
        self.qkv, self.dqkv = (torch.empty((batch, tokens, 3, model.heads, model.head_dim), **half) for _ in range(2))
        self.att = torch.empty(heads, **half)
        self.lse = torch.empty((batch, model.heads, tokens), device=dev)
        q, k, _ = self.qkv.unbind(2)
        fwd, bwd = dblp.dblp_attention_workspace_bytes(q, k, causal=True)
        ws = max(fwd, bwd, dblp.dblp_embed_grad_workspace_bytes(n, model.rows, d))
        self.ws = torch.empty(ws, dtype=torch.uint8, device=dev)

    def step(self, tokens, targets, step):
        """Loss of next-token prediction for int32 `tokens`, `targets` [batch, tokens]; leaves the gradient in self.grad."""
        m, n, d = self.model, tokens.numel(), self.model.width
        ids, want = tokens.reshape(-1), targets.reshape(-1).long()
        table, w_qkv, w_out = (w.bfloat16() for w in (m.table, m.w_qkv, m.w_out))
        q, k, v = self.qkv.unbind(2)

        dblp.dblp_embed(m.table, ids, self.emb, scale=math.sqrt(d))
        dblp.dblp_dropout(self.emb, self.x0, self.p, self.seed, step, EMBED_SITE)
        torch.mm(self.x0, w_qkv, out=self.qkv.view(n, 3 * d))
        dblp.dblp_attention(q, k, v, self.att, self.lse, self.ws, causal=True)
        y = torch.mm(self.att.view(n, d), w_out)
        dblp.dblp_dropout(y, self.x1, self.p, self.seed, step, RESIDUAL_SITE, residual=self.x0)
        logits = torch.mm(self.x1, table.t()).float()
        logp = torch.log_softmax(logits, dim=1)
        loss = -logp.gather(1, want[:, None]).mean()

        d_table, d_qkv, d_out = m.views(self.grad)
        dlogits = logp.exp()
        dlogits[torch.arange(n, device=ids.device), want] -= 1
        dlogits = dlogits.mul_(1.0 / n).bfloat16()
        d_table.copy_(torch.mm(dlogits.t(), self.x1))                     # the output layer's share of the tied table
        dx1 = torch.mm(dlogits, table)
        dy = y
        dblp.dblp_dropout_grad(dx1, dy, self.p, self.seed, step, RESIDUAL_SITE)
        d_out.copy_(torch.mm(self.att.view(n, d).t(), dy))
        datt = torch.mm(dy, w_out.t()).view(self.att.shape)
        dq, dk, dv = self.dqkv.unbind(2)
        dblp.dblp_attention_grad(q, k, v, self.att, datt, self.lse, dq, dk, dv, self.ws, causal=True)
        dqkv = self.dqkv.view(n, 3 * d)
        d_qkv.copy_(torch.mm(self.x0.t(), dqkv))
        torch.addmm(dx1, dqkv, w_qkv.t(), out=self.dx)
        dblp.dblp_dropout_grad(self.dx, self.dx, self.p, self.seed, step, EMBED_SITE)
        dblp.dblp_embed_grad(self.dx, ids, d_table, self.ws, scale=math.sqrt(d), accumulate=True)
        return loss


def train(rounds, workers=4, rows=512, heads=4, head_dim=64, batch=4, tokens=128, lr=0.5, loss=0.02, bound_ppm=50000, device="cuda:0"):
    """`rounds` rounds of data-parallel training over a lossy transport; returns the mean loss of each.  The task: the next
    token is a fixed permutation of the last one."""
    torch.cuda.set_device(device)
    model = TokenModel(rows, heads, head_dim, device)
    ws = [Worker(model, batch, tokens, seed=100 + w) for w in range(workers)]
    work = wl.Workload("worker", workers, "f32", 1408, model.numel, 0.0, wl.LossSpec("iid", loss), seed=7)
    plan = dblp.Plan(work.numel, work.dtype, work.payload_bytes, work.W)
    buf = plan.alloc_round(device)
    channel = dblp.loss_model(work.loss.kind, **work.loss.thresholds(plan.C))
    g = torch.Generator(device=device)
    g.manual_seed(1)
    follow = torch.randperm(rows, generator=g, device=device, dtype=torch.int32)
    losses, gave_up = [], dblp.dblp_wait_timeouts()
    for r in range(1, rounds + 1):
        seen = []
        for w in ws:
            x = torch.randint(0, rows, (batch, tokens), generator=g, device=device, dtype=torch.int32)
            seen.append(w.step(x, follow[x.long()], r))
        dblp.dblp_round_device(plan, [w.grad for w in ws], channel, work.seed, r, bound_ppm, dblp.DBLP_MEAN, buf)
        model.flat.add_(buf["agg"], alpha=-lr)                            # chunks that nobody delivered are zero: no change
        losses.append(torch.stack(seen).mean())
    out = [float(x) for x in losses]
    plan.close()
    if dblp.dblp_wait_timeouts() != gave_up:
        raise RuntimeError("a kernel gave up waiting: the gradients of some round are incomplete")
    return out


if __name__ == "__main__":
    for r, x in enumerate(train(60), 1):
        if r % 10 == 0 or r == 1:
            print("round %3d  loss %.4f" % (r, x))
