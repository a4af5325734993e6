"""A last partition of one layer over many classes: the losses that never keep its logits as a whole, and integers to serve it.

api.Segment's last layer holds the logits of a batch and their gradient; this one is trained on classes, or on the best few logits
of a teacher (the whole network, or one kept on another machine that sends no more than those), at sizes where those two would be
the largest things in memory.  Weights and biases are float32, bf16 copies of the weights enter the products, the update is torch's SGD.

Of api.Segment's calls the class has step, input_grad and forward, so it can be trained on the stored response of a left partition
(pipeline.train_epochs), be the frozen right partition of pipeline.recovery_epochs, and be joined (pipeline.joined_forward,
pipeline.accuracy).  forward computes in integers: it is the serving form.

A new layer is ready on every stream.  step, distil and refresh write the parameters and their copies (bf16, integers) on the current stream; input_grad and forward
only read them, on any number of streams at once, which wait for the last of those writes as for any tensor's.  All of these stay where they are for as long as the layer
lives, so that a captured call works on the parameters of the time of its replay; what a captured step calculates with besides, lr among it, is that of its capture.

    right = ClassLayer(width=512, classes=50000)
    losses = pipeline.train_epochs(right, stored, y, epochs=3, batch=1024)         # stored: bf16 [N, 512], y: int32 [N]
    top, ids = teacher.forward(x).topk(32, 1)                                      # another ClassLayer, say, on rows x
    loss = right.distil(x, top, ids, temperature=2.0)
"""

import torch

from . import api, datagen


class ClassLayer:
    """Logits x w^T + b of `classes` classes on rows of `width` bf16 values."""

    def __init__(self, width, classes, lr=0.01, momentum=0.9, seed=0, device="cuda"):
        self.widths, self.dtype = [width, classes], api.BF16
        (w, b), = datagen.uniform_weights(self.widths, seed)
        self.w, self.b = (torch.nn.Parameter(torch.from_numpy(a).to(device)) for a in (w, b))
        self.optimizer = torch.optim.SGD([self.w, self.b], lr=lr, momentum=momentum)
        if momentum:                       # from zeros the first step is like the others, also where it is a captured one
            for p in (self.w, self.b):
                self.optimizer.state[p]["momentum_buffer"] = torch.zeros_like(p.data)
        self.w16, self._w8 = self.w.data.bfloat16(), api.quantize_integers(self.w.data)
        torch.cuda.current_stream(self.w.device).synchronize()

    def refresh(self):
        """The copies of the weights that the products read, after the float32 ones have changed: here, not in the first call that needs them, whose stream others do not wait for."""
        self.w16.copy_(self.w.data)
        api.quantize_integers(self.w.data, out=self._w8)

    def _update(self, r):
        self.w.grad, self.b.grad = r.dw, r.dbias
        self.optimizer.step()
        self.refresh()

    def step(self, X, targets, want_loss=True, loss_out=None):
        """A training step against a class a row; returns the mean loss, a device scalar (written to loss_out as well where that is given)."""
        r = api.linear_cross_entropy(X, self.w16, targets, bias=self.b.data, dtype=api.F32)
        self._update(r)
        return r.loss if loss_out is None else loss_out.copy_(r.loss.reshape(loss_out.shape))

    def distil(self, X, top, classes, temperature=1.0):
        """A training step against a teacher's logits `top` of `classes` a row (api.linear_distillation); returns the mean loss."""
        r = api.linear_distillation(X, self.w16, top, classes, bias=self.b.data, temperature=temperature, dtype=api.F32)
        self._update(r)
        return r.loss

    def input_grad(self, X, targets, loss_out=None):
        """(gradient of X, mean loss); parameters untouched."""
        r = api.linear_cross_entropy(X, self.w16, targets, bias=self.b.data, weight_gradients=False)
        return r.dx, r.loss if loss_out is None else loss_out.copy_(r.loss.reshape(loss_out.shape))

    def forward(self, X, out=None):
        """The logits, in bf16 (or of out's type): rows and weights as integers with a scale each."""
        return api.product_integers(api.quantize_integers(X), self._w8, bias=self.b.data, out=out)
