"""A feed-forward sublayer of one rank, forward and backward, whole in the library's calls:

    z = x W1^T + b1 (kept in 8 bits),  g = gelu(z),  y = layer_norm(x + D(g W2^T + b2))

and from dy the gradients of x and of all parameters, written into a flat buffer that the reduce-scatter would read.  What is kept
between the passes is x, the norm's sum and statistics and the checkpoint of z: 1.06 bytes for each of its elements, where z and g
in 16 bits would be 4.  Run:  python -m paper_2205_00119_amd.examples.feed_forward [--rows 4096] [--hidden 5120]
"""
import argparse

import torch

import paper_2205_00119_amd as mics

BF16, F32 = mics.MICS_DTYPE_BF16, mics.MICS_DTYPE_F32
GELU = mics.MICS_ACT_GELU
EPS = 1e-5


class FeedForward:
    """Places of the parameters in the flat buffer, and the buffers of one micro-batch."""

    def __init__(self, rows, hidden, inner, drop, device="cuda:0"):
        self.rows, self.hidden, self.inner, self.drop = rows, hidden, inner, drop
        self.shapes = {"W1": (inner, hidden), "b1": (inner,), "W2": (hidden, inner), "b2": (hidden,), "weight": (hidden,),
                       "norm_bias": (hidden,)}
        self.offsets, at = {}, 0
        for name, shape in self.shapes.items():
            self.offsets[name] = at
            at += -(-torch.Size(shape).numel() // 8) * 8           # every tensor on 16 bytes
        self.numel = at
        b = dict(dtype=torch.bfloat16, device=device)
        f = dict(dtype=torch.float32, device=device)
        # kept for the backward pass
        self.sum, self.mean, self.rstd = torch.empty(rows, hidden, **b), torch.empty(rows, **f), torch.empty(rows, **f)
        self.codes = torch.empty(rows, inner, dtype=torch.int8, device=device)
        self.scales = torch.empty(mics.mics_checkpoint_scales(rows, inner), **f)
        # of use within a pass; one scratch serves all calls, which the stream orders
        self.y, self.out, self.dx = (torch.empty(rows, hidden, **b) for _ in range(3))
        self.g, self.dg = (torch.empty(rows, inner, **b) for _ in range(2))
        self.scratch_bytes = max([mics.mics_linear_workspace_bytes(rows, hidden, inner), mics.mics_linear_workspace_bytes(rows, inner, hidden)]
                                 + [mics.mics_column_workspace_bytes(rows, n) for n in (hidden, inner)])
        self.scratch = torch.empty(self.scratch_bytes, dtype=torch.uint8, device=device)

    def views(self, flat):
        return {n: flat[self.offsets[n]:self.offsets[n] + torch.Size(s).numel()].view(s) for n, s in self.shapes.items()}

    def _work(self):
        return dict(workspace=self.scratch, workspace_bytes=self.scratch_bytes)

    def forward(self, params, x, seed, offset):
        w, rows, h, i = self.views(params), self.rows, self.hidden, self.inner
        types = dict(dtype=BF16, param_dtype=BF16)
        mics.mics_linear(self.g, None, self.codes, self.scales, x, w["W1"], w["b1"], None, rows, h, i, act=GELU, **types, **self._work())
        mics.mics_linear(self.out, None, None, None, self.g, w["W2"], None, None, rows, i, h, act=mics.MICS_ACT_NONE, **types,
                         **self._work())
        mics.mics_dropout_add_layer_norm(self.y, self.sum, self.mean, self.rstd, self.out, w["b2"], x, w["weight"], w["norm_bias"], rows, h,
                                         eps=EPS, drop=self.drop, seed=seed, offset=offset, **types)
        return self.y

    def backward(self, params, grads, x, dy, seed, offset):
        """The gradient of x; those of the parameters are written into `grads`."""
        w, g, rows, h, i = self.views(params), self.views(grads), self.rows, self.hidden, self.inner
        out, dresidual = self.out, self.dx
        mics.mics_dropout_add_layer_norm_backward(
            out, dresidual, g["b2"], g["weight"], g["norm_bias"], dy, None, self.sum, self.mean, self.rstd, w["weight"], rows, h,
            drop=self.drop, seed=seed, offset=offset, dtype=BF16, param_dtype=BF16, grad_dtype=BF16, **self._work())
        # g again from the checkpoint, for the gradient of W2
        mics.mics_checkpoint_read(self.g, self.codes, self.scales, rows, i, act=GELU, dtype=BF16)
        mics.mics_linear_backward_weight(g["W2"], out, self.g, rows, i, h, dtype=BF16, grad_dtype=BF16, **self._work())
        mics.mics_linear_backward_input(self.dg, out, w["W2"], None, rows, i, h, dtype=BF16, **self._work())
        mics.mics_activation_backward(self.dg, g["b1"], self.dg, None, self.codes, self.scales, rows, i, act=GELU, dtype=BF16,
                                      grad_dtype=BF16, **self._work())
        mics.mics_linear_backward_weight(g["W1"], self.dg, x, rows, h, i, dtype=BF16, grad_dtype=BF16, **self._work())
        mics.mics_linear_backward_input(self.dx, self.dg, w["W1"], dresidual, rows, h, i, dtype=BF16, **self._work())
        return self.dx


def initial(layer, seed, device="cuda:0"):
    """Parameters of a fresh layer in bf16."""
    gen = torch.Generator(device=device).manual_seed(seed)
    flat = torch.zeros(layer.numel, device=device)
    for name, view in layer.views(flat).items():
        if name == "weight":
            view.fill_(1.0)
        elif view.dim() == 2:
            view.normal_(0.0, view.shape[1] ** -0.5, generator=gen)
    return flat.to(torch.bfloat16)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rows", type=int, default=4096, help="tokens of the micro-batch")
    ap.add_argument("--hidden", type=int, default=5120)
    ap.add_argument("--drop", type=float, default=0.1)
    ap.add_argument("--steps", type=int, default=10)
    args = ap.parse_args(argv)
    layer = FeedForward(args.rows, args.hidden, 4 * args.hidden, args.drop)
    params = initial(layer, 1)
    grads = torch.empty_like(params)
    gen = torch.Generator(device="cuda:0").manual_seed(2)
    x, dy = (torch.randn(args.rows, args.hidden, generator=gen, device="cuda:0").to(torch.bfloat16) for _ in range(2))
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for step in range(args.steps + 1):
        if step == 1:
            begin.record()
        layer.forward(params, x, 3, 0)
        layer.backward(params, grads, x, dy, 3, 0)
    end.record()
    torch.cuda.synchronize()
    ms = begin.elapsed_time(end) / args.steps
    flops = 6 * 2 * args.rows * args.hidden * 4 * args.hidden
    print(f"{ms:.3f} ms for forward and backward, {flops / ms / 1e9:.0f} TFLOP/s of products")
    return ms


if __name__ == "__main__":
    main()
