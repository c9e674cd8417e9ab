"""Training steps of a language model's last layer on one partition group, through the library's calls:

    parameter shards -> hierarchical gather -> forward (feed-forward sublayer, its epilogue of bias, dropout, residual and
    layer norm, token log probabilities) -> backward into the rank's flat gradient -> reduce-scatter-accumulate over the
    group's ranks and micro-steps -> scaling and Adam on every shard, which writes the shards of the next gather.

The p ranks of the group live on one GPU, each with its own tokens; matrix products are torch's.  The layer is
    u = x W1 + b1,  g = gelu(u),  y = layer_norm(x + D(g W2 + b2)),  logits = y E,
and learns to tell every token's successor.  Run:  python -m paper_2205_00119_amd.examples.train_layer [--steps 20]
"""
import argparse

import torch

import paper_2205_00119_amd as mics

BF16, F32 = mics.MICS_DTYPE_BF16, mics.MICS_DTYPE_F32
EPS = 1e-5


class Layer:
    """Shapes and places of the parameters in the flat buffer, and the buffers one rank's step needs."""

    def __init__(self, rows, hidden, inner, vocab, drop, device="cuda:0"):
        self.rows, self.hidden, self.inner, self.vocab, self.drop = rows, hidden, inner, vocab, drop
        self.shapes = {"W1": (hidden, inner), "b1": (inner,), "W2": (inner, hidden), "b2": (hidden,), "weight": (hidden,),
                       "norm_bias": (hidden,), "E": (hidden, vocab)}
        self.offsets, at = {}, 0
        for name, shape in self.shapes.items():
            self.offsets[name] = at
            at += -(-torch.Size(shape).numel() // 8) * 8           # every tensor on 16 bytes
        self.numel = at
        b = dict(dtype=torch.bfloat16, device=device)
        f = dict(dtype=torch.float32, device=device)
        self.y, self.sum, self.dx, self.dresidual = (torch.empty(rows, hidden, **b) for _ in range(4))
        self.mean, self.rstd, self.logprob, self.entropy, self.lse = (torch.empty(rows, **f) for _ in range(5))
        self.dlogprob = torch.full((rows,), -1.0 / rows, **f)      # the loss is the mean of -log p
        # one scratch for all backward passes: the stream orders them
        self.workspace_bytes = max(mics.mics_column_workspace_bytes(rows, n) for n in (hidden, inner))
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
        self.loss_bytes = mics.mics_token_logprobs_workspace_bytes(rows, vocab)
        self.loss_workspace = torch.empty(self.loss_bytes, dtype=torch.uint8, device=device)
        # how far apart the offsets of two calls of the generator have to be
        self.counters = mics.mics_dropout_counters(rows, hidden)

    def views(self, flat):
        return {n: flat[self.offsets[n]:self.offsets[n] + torch.Size(s).numel()].view(s) for n, s in self.shapes.items()}

    def step(self, params, grads, x, targets, seed, offset):
        """Loss of one micro-batch (a device scalar); its gradients are written into the flat buffer `grads`."""
        w, g = self.views(params), self.views(grads)
        rows, h, v = self.rows, self.hidden, self.vocab
        key = dict(drop=self.drop, seed=seed, offset=offset)
        types = dict(dtype=BF16, param_dtype=BF16)
        scratch = dict(grad_dtype=BF16, workspace=self.workspace, workspace_bytes=self.workspace_bytes)

        u = torch.mm(x, w["W1"])
        mics.mics_bias_dropout_add(u, u, w["b1"], None, rows, self.inner, drop=0.0, seed=0, offset=0, **types)
        act = torch.nn.functional.gelu(u)
        out = torch.mm(act, w["W2"])
        mics.mics_dropout_add_layer_norm(self.y, self.sum, self.mean, self.rstd, out, w["b2"], x, w["weight"], w["norm_bias"], rows, h,
                                         eps=EPS, **key, **types)
        logits = torch.mm(self.y, w["E"])
        mics.mics_token_logprobs(self.logprob, self.entropy, self.lse, None, None, logits, targets, rows, v, dtype=BF16,
                                 workspace=self.loss_workspace, workspace_bytes=self.loss_bytes)
        loss = -self.logprob.mean()

        # backward: the logits' gradient takes their place
        mics.mics_token_logprobs_backward(logits, logits, targets, self.lse, None, self.dlogprob, None, rows, v, dtype=BF16)
        torch.mm(self.y.t(), logits, out=g["E"])
        dy = torch.mm(logits, w["E"].t())
        mics.mics_dropout_add_layer_norm_backward(
            self.dx, self.dresidual, g["b2"], g["weight"], g["norm_bias"], dy, None, self.sum, self.mean, self.rstd, w["weight"], rows, h,
            **key, **types, **scratch)
        torch.mm(act.t(), self.dx, out=g["W2"])
        du = torch.ops.aten.gelu_backward(torch.mm(self.dx, w["W2"].t()), u)
        mics.mics_bias_dropout_add_backward(du, g["b1"], du, rows, self.inner, drop=0.0, seed=0, offset=0, dtype=BF16, **scratch)
        torch.mm(x.t(), du, out=g["W1"])
        return loss


class Group:
    """A partition group of p ranks (k on a node): master shards, Adam states and the stage-1 buffers of the gather."""

    def __init__(self, layer, p, k, seed, lr, device="cuda:0"):
        self.layer, self.p, self.k, self.lr, self.steps = layer, p, k, lr, 0
        self.S = S = mics.mics_shard_elems(layer.numel, p, 8)
        gen = torch.Generator(device=device).manual_seed(seed)
        flat = torch.zeros(p * S, device=device)
        for name, view in layer.views(flat).items():
            if name == "weight":
                view.fill_(1.0)
            elif view.dim() == 2:
                view.normal_(0.0, 0.02 if name != "E" else 0.05, generator=gen)
        self.master = [flat[r * S:(r + 1) * S].clone() for r in range(p)]
        self.m, self.v = ([torch.zeros(S, device=device) for _ in range(p)] for _ in range(2))
        # rank r = j k + l leaves its 16-bit shard in slot j of the stage-1 buffer of local rank l
        self.stage1 = [torch.empty(p // k * S, dtype=torch.bfloat16, device=device) for _ in range(k)]
        for r in range(p):
            self.slot(r).copy_(self.master[r])
        self.params = torch.empty(layer.numel, dtype=torch.bfloat16, device=device)
        self.grads = [torch.zeros(p * S, dtype=torch.bfloat16, device=device) for _ in range(p)]
        self.acc = [torch.empty(S, device=device) for _ in range(p)]

    def slot(self, r):
        j, l = divmod(r, self.k)
        return self.stage1[l][j * self.S:(j + 1) * self.S]

    def train_step(self, batches, seed):
        """One step over micro-batches [[(x, targets) of every rank], ...]; returns the mean loss."""
        layer, p, S = self.layer, self.p, self.S
        losses = []
        for t, micro in enumerate(batches):
            mics.mics_hier_gather_reorder(self.params, self.stage1, layer.numel, S, p, self.k, 2)
            for r, (x, targets) in enumerate(micro):
                call = (self.steps * len(batches) + t) * p + r
                losses.append(layer.step(self.params, self.grads[r], x, targets, seed, call * layer.counters))
            for r in range(p):
                mics.mics_reduce_scatter_accum(self.acc[r], self.grads, r * S, S, t > 0)
        self.steps += 1
        for r in range(p):
            mics.mics_replica_average_adam_shard(self.master[r], self.m[r], self.v[r], self.slot(r), [self.acc[r]], S,
                                                 1.0 / (p * len(batches)), lr=self.lr, beta1=0.9, beta2=0.98, eps=1e-8,
                                                 weight_decay=0.0, step=self.steps)
        return torch.stack(losses).mean()


def batches_of(layer, p, s, gen, table, embedding):
    """Tokens whose successors a fixed table gives, as the embeddings the layer below would hand over."""
    out = []
    for _ in range(s):
        micro = []
        for _ in range(p):
            tokens = torch.randint(0, layer.vocab, (layer.rows,), generator=gen, device=table.device)
            micro.append((embedding[tokens], table[tokens]))
        out.append(micro)
    return out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--rows", type=int, default=512, help="tokens of a rank's micro-batch")
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--ranks", type=int, default=4, help="of the partition group, two on a node")
    ap.add_argument("--micro-steps", type=int, default=2)
    ap.add_argument("--drop", type=float, default=0.1)
    ap.add_argument("--lr", type=float, default=2e-3)
    args = ap.parse_args(argv)
    device = "cuda:0"
    gen = torch.Generator(device=device).manual_seed(1)
    layer = Layer(args.rows, args.hidden, 4 * args.hidden, args.vocab, args.drop)
    group = Group(layer, args.ranks, 2, 2, args.lr)
    table = torch.randperm(args.vocab, generator=gen, device=device)
    embedding = torch.randn(args.vocab, args.hidden, generator=gen, device=device).to(torch.bfloat16)
    losses = []
    for step in range(args.steps):
        loss = group.train_step(batches_of(layer, args.ranks, args.micro_steps, gen, table, embedding), seed=3)
        losses.append(float(loss))
        print(f"step {step + 1:3d}  loss {losses[-1]:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    main()
