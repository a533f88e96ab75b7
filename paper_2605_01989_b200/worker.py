"""A worker's training step on the library's own operators, and rounds of it through the server path (Algorithm 4: compute
the gradient, send it, receive the mean, update).

The model is the smallest one that meets all of them: token embedding, dropout, one causal attention block with a residual
dropout, and an output layer tied to the embedding table.  Plain matrix products are torch's; embedding, dropout, attention
and their gradients are the library's.  The gradient is written straight into one flat buffer in the order of the plan's
tensors, which is what dblp_packetize reads.

A second model is a whole decoder block: projections, norm and rotation of queries and keys, attention, a feed-forward layer, all
its products, epilogues and gradients the library's, and its matrices updated by the orthogonalised mean of a round.

    python -m paper_2605_01989_b200.worker          # four workers, 2 % of the packets lost, a few rounds
    python -m paper_2605_01989_b200.worker block    # the same with the decoder block
"""
import math
import sys

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

    def update(self, mean, lr):
        self.flat.add_(mean, alpha=-lr)                   # chunks that nobody delivered are zero: no change


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


class BlockModel:
    """A decoder block in fp32 in one flat vector: table, qkv, the norms' weights, output, up (with bias), down (with bias)."""

    NAMES = ("table", "w_qkv", "q_norm", "k_norm", "w_out", "w_up", "b_up", "w_down", "b_down")
    MATRICES = ("w_qkv", "w_out", "w_up", "w_down")       # updated by their orthogonalised momentum

    def __init__(self, rows, heads, head_dim, device, seed=0, theta=10000.0):
        self.rows, self.heads, self.head_dim, self.width = rows, heads, head_dim, heads * head_dim
        d = self.width
        self.shapes = [(rows, d), (d, 3 * d), (head_dim,), (head_dim,), (d, d), (d, 4 * d), (4 * d,), (4 * d, d), (d,)]
        self.numel = [math.prod(s) for s in self.shapes]
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.flat = torch.randn(sum(self.numel), generator=g, device=device) * 0.02
        self.momentum = torch.zeros_like(self.flat)
        params = self.views(self.flat)
        for name in ("q_norm", "k_norm"):
            params[name].fill_(1.0)
        self.freqs = theta ** (-torch.arange(head_dim // 2, device=device, dtype=torch.float64) * 2 / head_dim)
        self.turned = {n: torch.empty(params[n].shape, dtype=torch.bfloat16, device=device) for n in self.MATRICES}
        need = max(dblp.dblp_orthogonalize_workspace_bytes(params[n], self.turned[n]) for n in self.MATRICES)
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)

    def views(self, flat):
        """The tensors of a flat vector laid out like the parameters, by name."""
        return {n: v.view(s) for n, v, s in zip(self.NAMES, flat.split(self.numel), self.shapes)}

    def update(self, mean, lr, mu=0.9):
        """Momentum of the round's mean; matrices move by it with its singular values near 1, the rest as it is."""
        self.momentum.mul_(mu).add_(mean)
        params, momentum = self.views(self.flat), self.views(self.momentum)
        for n, w in params.items():
            if n in self.turned:
                scale = math.sqrt(max(1.0, w.shape[0] / w.shape[1]))
                dblp.dblp_orthogonalize(momentum[n], self.turned[n], self.ws, scale=scale)
                w.add_(self.turned[n], alpha=-0.02 * lr)
            else:
                w.add_(momentum[n], alpha=-lr)


class BlockWorker:
    """One worker of a BlockModel: buffers for `batch` sequences of `tokens` tokens, and its flat fp32 gradient."""

    def __init__(self, model, batch, tokens, seed=0):
        self.model = model
        dev, d, n, H, D = model.flat.device, model.width, batch * tokens, model.heads, model.head_dim
        half = dict(dtype=torch.bfloat16, device=dev)
        heads = (batch, tokens, H, D)
        self.positions = torch.arange(tokens, device=dev, dtype=torch.int32).expand(batch, tokens)
        self.grad = torch.zeros(sum(model.numel), device=dev)
        self.x0, self.x1, self.x2, self.dx0, self.dx1, self.dx2 = (torch.empty((n, d), **half) for _ in range(6))
        self.qkv, self.dqkv = (torch.empty((batch, tokens, 3, H, D), **half) for _ in range(2))
        self.q, self.k, self.att, self.dq, self.dk, self.datt = (torch.empty(heads, **half) for _ in range(6))
        self.lse = torch.empty((batch, H, tokens), device=dev)
        self.pre, self.mid, self.dpre = (torch.empty((n, 4 * d), **half) for _ in range(3))
        self.logits = torch.empty((n, model.rows), device=dev)
        w = {name: t.bfloat16() for name, t in model.views(model.flat).items()}
        dlogits = self.logits.bfloat16()
        layers = [(self.x0, w["w_qkv"], self.qkv.view(n, 3 * d)), (self.att.view(n, d), w["w_out"], self.x1), (self.x1, w["w_up"], self.pre),
                  (self.mid, w["w_down"], self.x2), (self.x2, w["table"].t(), dlogits)]
        need = [b for layer in layers for b in dblp.dblp_linear_workspace_bytes(*layer)]
        need += dblp.dblp_attention_workspace_bytes(self.q, self.k, causal=True)
        need += [dblp.dblp_embed_grad_workspace_bytes(n, model.rows, d), dblp.dblp_norm_rotate_grad_workspace_bytes(self.q, self.k)]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device=dev)

    def step(self, tokens, targets, step):
        """Loss of next-token prediction for int32 `tokens`, `targets` [batch, tokens]; leaves the gradient in self.grad."""
        m, n, d, ws = self.model, tokens.numel(), self.model.width, self.ws
        ids, want = tokens.reshape(-1), targets.reshape(-1).long()
        p = m.views(m.flat)
        w = {name: p[name].bfloat16() for name in ("table",) + m.MATRICES}
        q, k, v = self.qkv.unbind(2)
        att = self.att.view(n, d)

        dblp.dblp_embed(p["table"], ids, self.x0, scale=math.sqrt(d))
        dblp.dblp_linear(self.x0, w["w_qkv"], self.qkv.view(n, 3 * d), ws)
        dblp.dblp_norm_rotate(q, k, p["q_norm"], p["k_norm"], self.positions, m.freqs, self.q, self.k)
        dblp.dblp_attention(self.q, self.k, v, self.att, self.lse, ws, causal=True)
        dblp.dblp_linear(att, w["w_out"], self.x1, ws, residual=self.x0)
        dblp.dblp_linear(self.x1, w["w_up"], self.mid, ws, bias=p["b_up"], pre=self.pre, activation="gelu")
        dblp.dblp_linear(self.mid, w["w_down"], self.x2, ws, bias=p["b_down"], residual=self.x1)
        dblp.dblp_linear(self.x2, w["table"].t(), self.logits, ws)
        logp = torch.log_softmax(self.logits, dim=1)
        loss = -logp.gather(1, want[:, None]).mean()

        g = m.views(self.grad)
        dlogits = logp.exp()
        dlogits[torch.arange(n, device=ids.device), want] -= 1
        dlogits = dlogits.mul_(1.0 / n).bfloat16()
        dblp.dblp_linear_grad(dlogits, self.x2, w["table"].t(), dx=self.dx2, dw=g["table"].t(), ws=ws)
        dblp.dblp_linear_grad(self.dx2, self.mid, w["w_down"], dx=self.dpre, dw=g["w_down"], dbias=g["b_down"], ws=ws, pre=self.pre,
                              activation="gelu")
        dblp.dblp_linear_grad(self.dpre, self.x1, w["w_up"], dx=self.dx1, dw=g["w_up"], dbias=g["b_up"], ws=ws, residual=self.dx2)
        dblp.dblp_linear_grad(self.dx1, att, w["w_out"], dx=self.datt.view(n, d), dw=g["w_out"], ws=ws)
        dq, dk, dv = self.dqkv.unbind(2)
        dblp.dblp_attention_grad(self.q, self.k, v, self.att, self.datt, self.lse, self.dq, self.dk, dv, ws, causal=True)
        dblp.dblp_norm_rotate_grad(q, k, p["q_norm"], p["k_norm"], self.positions, m.freqs, self.dq, self.dk, dq, dk, g["q_norm"],
                                   g["k_norm"], ws)
        dblp.dblp_linear_grad(self.dqkv.view(n, 3 * d), self.x0, w["w_qkv"], dx=self.dx0, dw=g["w_qkv"], ws=ws, residual=self.dx1)
        dblp.dblp_embed_grad(self.dx0, ids, g["table"], ws, scale=math.sqrt(d), accumulate=True)
        return loss


def train(rounds, workers=4, rows=512, heads=4, head_dim=64, batch=4, tokens=128, lr=0.5, loss=0.02, bound_ppm=50000, device="cuda:0",
          block=False):
    """`rounds` rounds of data-parallel training over a lossy transport; returns the mean loss of each.  The task: the next
    token is a fixed permutation of the last one.  With `block` the model is the decoder block."""
    torch.cuda.set_device(device)
    model = (BlockModel if block else TokenModel)(rows, heads, head_dim, device)
    ws = [(BlockWorker if block else Worker)(model, batch, tokens, seed=100 + w) for w in range(workers)]
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
        model.update(buf["agg"], lr)
        losses.append(torch.stack(seen).mean())
    out = [float(x) for x in losses]
    plan.close()
    if dblp.dblp_wait_timeouts() != gave_up:
        raise RuntimeError("a kernel gave up waiting: the gradients of some round are incomplete")
    return out


if __name__ == "__main__":
    for r, x in enumerate(train(60, block="block" in sys.argv[1:]), 1):
        if r % 10 == 0 or r == 1:
            print("round %3d  loss %.4f" % (r, x))
