"""A residual segment in 8 bits: the operators of the library put together as a left partition.

Blocks of   h <- h + W2 relu(W1 norm(h) + b1) + b2   on rows of one width.  The normalised rows, the hidden activations, both
weight matrices and every gradient that enters a product are 8-bit matrices (api.Quantized); h, the gradients between
blocks and the outputs of products are bf16, weights and their gradients float32.  Gradients are clipped together by
their norm before the update, which is torch's SGD on the float32 weights.

Of api.Segment's calls the class has forward and step_external, so it can be trained through a frozen right partition (Sec. 5
of the paper, pipeline.recovery_epochs), joined with it (pipeline.joined_forward, pipeline.accuracy) and its response stored
(pipeline.store_response).  It has no step against labels, which pipeline.train_epochs, train_partitioned and train_simultaneous call:

    left = ResidualSegment(width=512, hidden=2048, blocks=2)
    right = api.Segment([512, 1024, 47], api.RELU_HIDDEN_IDENTITY_LAST, api.SOFTMAX_XENT, max_batch=256, dtype=api.BF16, input_grad=True)
    right.init(1)
    losses = pipeline.recovery_epochs(left, right, X, y, epochs=3, batch=256)      # X: bf16 [N, 512], y: int32 [N]
"""

import torch

from . import api, datagen


class _Block:
    def __init__(self, width, hidden, seed, device):
        (w1, b1), (w2, b2) = datagen.uniform_weights([width, hidden, width], seed)
        up = lambda a: torch.nn.Parameter(torch.from_numpy(a).to(device))  # noqa: E731
        self.gamma = torch.nn.Parameter(torch.ones(width, device=device))
        self.w1, self.b1, self.w2, self.b2 = up(w1), up(b1), up(w2), up(b2)
        self.refresh()

    def parameters(self):
        return [self.gamma, self.w1, self.b1, self.w2, self.b2]

    def refresh(self):
        """The weights in 8 bits, as they are for the forward products and transposed for the gradients of their inputs."""
        self.w1_8 = api.quantize(self.w1.data, block=128, transposed=True)
        self.w2_8 = api.quantize(self.w2.data, block=128, transposed=True)

    def forward(self, h, f, eps, keep):
        """From the sum so far as h + f (f may be None): (the sum, what the block adds to it, what its backward pass needs)."""
        n = api.rmsnorm(h if f is None else f, self.gamma.data, residual=None if f is None else h, eps=eps, normed=keep)
        z = api.product(n.y8, self.w1_8.rows, bias=self.b1.data, relu=True)
        f = api.product(api.quantize(z).rows, self.w2_8.rows, bias=self.b2.data)
        return n.h, f, (n, z) if keep else None

    def backward(self, d, kept):
        """From the gradient of the sum behind the block: (that of the sum in front of it, those of the parameters)."""
        n, z = kept
        df = api.quantize(d, transposed=True, column_sums=True)
        da = api.product(df.rows, self.w2_8.transposed)
        dw2 = api.product(df.transposed, api.quantize(z, rows=False, transposed=True).transposed, dtype=api.F32)
        dz = api.quantize(da, transposed=True, mask=z, column_sums=True)
        dy = api.product(dz.rows, self.w1_8.transposed)
        dw1 = api.product(dz.transposed, api.quantize(n.y, rows=False, transposed=True).transposed, dtype=api.F32)
        dx, dgamma = api.rmsnorm_backward(dy, n.h, self.gamma.data, n.rstd, dh=d)
        return dx, [dgamma, dw1, dz.column_sums, dw2, df.column_sums]


class ResidualSegment:
    """`blocks` residual blocks on rows of `width` bf16 values, each with a hidden layer of `hidden`."""

    def __init__(self, width, hidden, blocks, lr=0.01, momentum=0.9, max_norm=1.0, eps=1e-6, seed=0, device="cuda"):
        self.widths, self.dtype, self.eps, self.max_norm = [width, width], api.BF16, eps, max_norm
        self.blocks = [_Block(width, hidden, seed + i, device) for i in range(blocks)]
        self.parameters = [p for b in self.blocks for p in b.parameters()]
        self.optimizer = torch.optim.SGD(self.parameters, lr=lr, momentum=momentum)
        self.gradient_norm = None          # of the last step, before clipping: a device scalar

    def _forward(self, X, keep):
        assert X.dtype is torch.bfloat16 and X.dim() == 2 and X.size(1) == self.widths[0]
        h, f, kept = X, None, []
        for b in self.blocks:
            h, f, k = b.forward(h, f, self.eps, keep)
            kept.append(k)
        return api.rmsnorm(f, residual=h, eps=self.eps, quantized=False).h, kept

    def forward(self, X, out=None):
        r, _ = self._forward(X, False)
        return r if out is None else out.copy_(r)

    def backward(self, X, dA_out):
        """(gradient of X, gradients of self.parameters) for the gradient of the output."""
        _, kept = self._forward(X, True)
        d, grads = dA_out, []
        for b, k in zip(reversed(self.blocks), reversed(kept)):
            d, g = b.backward(d, k)
            grads = g + grads
        return d, grads

    def step_external(self, X, dA_out):
        """A training step from the gradient of the segment's output; a step whose gradients are not finite changes nothing."""
        _, grads = self.backward(X, dA_out)
        self.gradient_norm = api.clip_gradients(grads, self.max_norm)
        if not bool(torch.isfinite(self.gradient_norm)):
            return
        for p, g in zip(self.parameters, grads):
            p.grad = g
        self.optimizer.step()
        for b in self.blocks:
            b.refresh()
