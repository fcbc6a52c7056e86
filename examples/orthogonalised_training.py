"""Training with orthogonalised updates, on synthetic images.

    python examples/orthogonalised_training.py              # both networks, loss every ten steps

`FeedForward`: a residual feed-forward classifier made of linear layers.  Images arrive as encoded 8-bit pixels, the decode layer
turns them into 16-bit rows, every layer is one `linear_forward` with its activation and skip connection, every gradient one
`linear_backward` that writes into a flat vector, and all weight matrices are updated by one `muon_update`.

`train_cnn`: the checkpointed training step of a CNN gives the gradients; its convolution and linear weights are matrices of the flat
parameter vector and take the same update, the other parameters plain steps.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2105_00619_amd import binding as B  # noqa: E402
from paper_2105_00619_amd import workloads as W  # noqa: E402


class FeedForward:
    """h = gelu(x W_in^T + b);  h = h + W_down gelu(W_up h + b) + b for every block;  logits = h W_out^T + b.

    The fp32 masters of all matrices lie in one flat vector, their 16-bit copies, gradients and momenta in vectors like it."""

    def __init__(self, features, width, hidden, blocks, classes, dtype=torch.bfloat16, seed=0):
        self.shapes = [(width, features)] + [(hidden, width), (width, hidden)] * blocks + [(classes, width)]
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.w = torch.cat([torch.randn(r * c, generator=gen, device="cuda") * c ** -0.5 for r, c in self.shapes])
        self.w16, self.v = self.w.to(dtype), torch.zeros_like(self.w)
        self.g = torch.zeros_like(self.w16)
        self.ortho = B.Orthogonalizer(self.shapes)
        self.weights, self.dweights = self._views(self.w16), self._views(self.g)
        outs = [r for r, _ in self.shapes]
        self.b, self.db = torch.zeros(sum(outs), device="cuda"), torch.zeros(sum(outs), device="cuda")
        self.biases, self.dbiases = self.b.split(outs), self.db.split(outs)
        self.skipped = torch.zeros(1, dtype=torch.int32, device="cuda")

    def _views(self, flat):
        return [p.view(r, c) for p, (r, c) in zip(flat.split([r * c for r, c in self.shapes]), self.shapes)]

    def forward(self, x):
        """The logits, and what the gradients need: input and pre-activation of every layer."""
        last, kept = len(self.shapes) - 1, []
        h = skip = x
        for i, (w, b) in enumerate(zip(self.weights, self.biases)):
            down = 0 < i < last and i % 2 == 0
            if not down:
                skip = h
            if down or i == last:  # no activation; the end of a block adds what the block began with
                y, z = B.linear_forward(h, w, b, residual=skip if down else None), None
            else:
                y, z = B.linear_forward(h, w, b, activation="gelu", save_pre=True)
            kept.append((h, z))
            h = y
        return h, kept

    def backward(self, d, kept):
        """All gradients from d, the gradient of the logits, into self.g and self.db."""
        last = len(self.shapes) - 1
        skip = None  # the gradient that passes a block by
        for i in range(last, -1, -1):
            x, z = kept[i]
            if 0 < i < last and i % 2 == 0:
                skip = d
            dx, _, _ = B.linear_backward(d, x, self.weights[i], z, activation="none" if z is None else "gelu",
                                         need=("dx", "dw", "dbias") if i else ("dw", "dbias"), dw=self.dweights[i], dbias=self.dbiases[i])
            if 0 < i < last and i % 2 == 1:
                dx = dx + skip
            d = dx

    def step(self, x, y, lr):
        logits, kept = self.forward(x)
        p = torch.log_softmax(logits.float(), 1)
        loss = -p.gather(1, y[:, None]).mean()
        d = (p.exp() - torch.nn.functional.one_hot(y, p.shape[1])) / len(y)
        self.backward(d.to(x.dtype), kept)
        self.ortho.muon_update(self.w, self.v, self.g, lr=lr, weight_decay=0.01, weights16=self.w16, skipped=self.skipped)
        self.b.sub_(torch.where(self.skipped == 0, lr * self.db, 0.0))  # (not 0 times what may be infinite)
        return loss


def train_feed_forward(steps=60, batch=256, size=16, classes=10, width=256, hidden=1024, blocks=2, lr=0.02, report=None):
    """The loss of every step on one batch of encoded images."""
    pixels = torch.from_numpy(W.make_pixels_u8(batch, size, size, 3)).cuda()
    z = 16
    encoded = B.encode(pixels, z)
    x = B.decode_normalized(encoded, batch, size * size * 3, z, 3, [4 / 255.0] * 3, [-2.0] * 3, W.BF16).view(batch, -1)
    y = torch.from_numpy(W.make_labels(batch, classes)).long().cuda()
    net = FeedForward(x.shape[1], width, hidden, blocks, classes)
    losses = []
    for i in range(steps):
        losses.append(net.step(x, y, lr))
        if report and i % 10 == 0:
            report("feed-forward", i, float(losses[-1]))
    return [float(v) for v in losses]


def train_cnn(steps=30, batch=64, size=16, classes=10, lr=0.02, report=None):
    """The same for a residual CNN: gradients of the checkpointed step, weights of every layer orthogonalised as C_out x (k k C_in)."""
    units = W.resnet_basic([1, 1], classes, base=16)
    t = B.SeqTrainer(units, k_segments=2, precision=W.BF16, batch=batch, height=size, width=size, channels=3, num_classes=classes)
    w = torch.from_numpy(W.make_params(units, size, size)).cuda()
    matrices, other, at = [], torch.ones_like(w, dtype=torch.bool), 0
    for _, shape, role, _ in W.param_layout(units, size, size):
        rows, cols = shape[0], 1
        for n in shape[1:]:
            cols *= n
        if role in ("conv_w", "lin_w"):
            matrices.append((at, rows, cols, cols))
            other[at:at + rows * cols] = False
        at += rows * cols
    ortho = B.Orthogonalizer(matrices)
    v, g = torch.zeros_like(w), torch.zeros_like(w)
    x = torch.from_numpy(W.make_images(batch, size, size, 3)).cuda()
    y = torch.from_numpy(W.make_labels(batch, classes)).cuda()
    losses = []
    t.set_params(w)
    for i in range(steps):
        step = t.step(x, y, lr=0.0, grads=g)
        losses.append(step["loss"])
        if not step["skipped"]:  # (else g holds no gradient)
            ortho.muon_update(w, v, g, lr=lr)
            w.sub_(torch.where(other, lr * g, 0.0))
            t.update_params(w)
        if report and i % 10 == 0:
            report("cnn", i, losses[-1])
    return losses


if __name__ == "__main__":
    def say(name, i, loss):
        print("%-12s step %3d  loss %.4f" % (name, i, loss), flush=True)

    train_feed_forward(report=say)
    train_cnn(report=say)
