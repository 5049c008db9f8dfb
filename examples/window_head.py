"""A trained head over ROCKET features of windows, and its use window by window.

Long series are cut into windows; the transform gives every window a feature
row, so that a series is a sequence of rows.  The head normalises each row by
groups, projects it, mixes the rows over time with a gated recurrence, joins
dropout of the result to the projection and classifies the mean over a series'
own windows.  After training, the same head follows streams: one window at a
time, the recurrence's state carried along.

    python examples/window_head.py            (a few seconds on one GPU)
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2601_17091_amd as rk  # noqa: E402
from paper_2601_17091_amd import sequence  # noqa: E402
from paper_2601_17091_amd.workloads import make_series  # noqa: E402


class GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, activation):
        y, mean, rstd = sequence.group_norm(x, groups, weight, bias, activation=activation)
        ctx.save_for_backward(x, mean, rstd, weight, bias)
        ctx.kind = groups, activation
        return y

    @staticmethod
    def backward(ctx, dy):
        x, mean, rstd, weight, bias = ctx.saved_tensors
        groups, activation = ctx.kind
        dx, dweight, dbias = sequence.group_norm_backward(dy.contiguous(), x, groups, mean, rstd, weight, bias,
                                                          activation=activation)
        return dx, dweight, dbias, None, None


class Recurrence(torch.autograd.Function):
    """On a projection [n, steps, 3 D] whose blocks are v, f and o."""

    @staticmethod
    def forward(ctx, p, lengths):
        v, f, o = p.chunk(3, dim=2)
        y, _, states = sequence.recurrence(v, f, o, lengths=lengths, keep_states=True)
        ctx.save_for_backward(p, states, lengths)
        return y

    @staticmethod
    def backward(ctx, dy):
        p, states, lengths = ctx.saved_tensors
        v, f, o = p.chunk(3, dim=2)
        dp = torch.empty_like(p)   # the three gradients, where the projection's is wanted
        sequence.recurrence_backward(dy.contiguous(), v, f, states, o, lengths=lengths, out=dp.chunk(3, dim=2))
        return dp, None


class Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, call):
        ctx.draw = p, seed, call
        return sequence.dropout(x, p, seed, call, residual=residual)

    @staticmethod
    def backward(ctx, dy):
        dy = dy.contiguous()
        return sequence.dropout_backward(dy, *ctx.draw), dy, None, None, None


class Head(torch.nn.Module):
    def __init__(self, features: int, groups: int, width: int, classes: int, p: float = 0.1, seed: int = 1):
        super().__init__()
        self.groups, self.width, self.p, self.seed = groups, width, p, seed
        self.weight = torch.nn.Parameter(torch.ones(features))
        self.bias = torch.nn.Parameter(torch.zeros(features))
        self.project = torch.nn.Linear(features, 3 * width)
        self.classify = torch.nn.Linear(width, classes)

    def rows(self, x):
        """Projections of feature rows [..., features], each row normalised by itself."""
        y = GroupNorm.apply(x.reshape(-1, 1, x.shape[-1]), self.weight, self.bias, self.groups, "silu")
        return self.project(y.reshape(x.shape))

    def forward(self, x, lengths, call: int = 0):
        """Logits [n, classes] of sequences [n, windows, features] of the given lengths."""
        p = self.rows(x)
        y, v = Recurrence.apply(p, lengths), p[:, :, :self.width]
        y = Dropout.apply(y, v, self.p, self.seed, call) if self.training else y + v
        own = torch.arange(x.shape[1], device=x.device)[None, :] < lengths[:, None]
        return self.classify((y * own[:, :, None]).sum(1) / lengths.clamp(min=1)[:, None])

    @torch.no_grad()
    def step(self, x, h):
        """One more window of every stream: x [n, features], state h [n, width], updated in place."""
        v, f, o = self.rows(x).chunk(3, dim=1)
        y, _ = sequence.recurrence_step(v, f, h, o, h_out=h)
        return y + v


def feature_sequences(plan, series, window: int, hop: int):
    """[n, windows, features] of series [n, steps]."""
    cut = series.unfold(1, hop if hop > window else window, hop)[:, :, :window].contiguous()
    n, windows, _ = cut.shape
    return plan.transform(cut.view(n * windows, window)).view(n, windows, -1)


def data(n: int, steps: int, seed: int):
    """Two kinds of series in turn, and their labels."""
    kinds = ("ar1", "sinusoids")
    x = torch.empty(n, steps)
    for k, kind in enumerate(kinds):
        x[k::2] = torch.from_numpy(make_series(kind, len(x[k::2]), steps, seed + k))
    return x.cuda(), (torch.arange(n) % 2).cuda()


def main(n: int = 64, steps: int = 4000, window: int = 128, kernels: int = 500, width: int = 64, epochs: int = 40,
         say=print):
    """Trains; returns the losses, the accuracy on new series, and how far the
    step by step states' mean is from the sequences'."""
    torch.manual_seed(0)
    plan = rk.Plan(rk.generate_kernels(201, kernels, window), window)
    series, labels = data(n, steps, 101)
    x = feature_sequences(plan, series, window, window)
    # recordings of unequal lengths
    lengths = torch.randint(1, x.shape[1] + 1, (n,), generator=torch.Generator().manual_seed(3)).int().cuda()
    head = Head(x.shape[2], 20, width, 2).cuda()
    adam = torch.optim.Adam(head.parameters(), lr=2e-3)
    losses = []
    for epoch in range(epochs):
        loss = torch.nn.functional.cross_entropy(head(x, lengths, call=epoch), labels)
        adam.zero_grad()
        loss.backward()
        adam.step()
        losses.append(float(loss.detach()))
        if epoch % 5 == 4:
            say("epoch %2d  loss %.4f" % (epoch + 1, losses[-1]))

    head.eval()
    series, labels = data(n, steps, 301)
    x = feature_sequences(plan, series, window, window)
    lengths = torch.full((n,), x.shape[1], dtype=torch.int32, device="cuda")
    with torch.no_grad():
        logits = head(x, lengths)
    accuracy = float((logits.argmax(1) == labels).float().mean())
    # the same series as streams
    h, total = torch.zeros(n, width, device="cuda"), torch.zeros(n, width, device="cuda")
    for t in range(x.shape[1]):
        total += head.step(x[:, t].contiguous(), h)
    with torch.no_grad():
        apart = float((head.classify(total / x.shape[1]) - logits).abs().max())
    say("accuracy on new series %.3f, logits of streams and of sequences apart by %.2g" % (accuracy, apart))
    return losses, accuracy, apart


if __name__ == "__main__":
    main()
