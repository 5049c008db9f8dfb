"""The example of a head over windows' features: the transform, group norm,
recurrence and dropout in one training loop, then window by window."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_window_head_trains_and_follows_streams():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import window_head
    finally:
        sys.path.pop(0)
    losses, accuracy, apart = window_head.main(say=lambda s: print(s, flush=True))
    assert losses[-1] < 0.5 * losses[0]
    assert accuracy > 0.9
    # fp32 sums of 31 windows in another order: rounding only
    assert apart < 1e-4


def test_window_head_gradients_against_plain_torch():
    """One step's gradients against autograd through elementary operations."""
    import torch

    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import window_head
    finally:
        sys.path.pop(0)
    torch.manual_seed(1)
    n, T, F, D = 5, 9, 60, 16
    head = window_head.Head(F, 6, D, 3, p=0.0).cuda()
    with torch.no_grad():
        head.weight.add_(0.2 * torch.randn(F, device="cuda"))
        head.bias.add_(0.2 * torch.randn(F, device="cuda"))
    x = torch.randn(n, T, F, device="cuda")
    lengths = torch.tensor([9, 1, 4, 9, 0], dtype=torch.int32, device="cuda")
    labels = torch.tensor([0, 1, 2, 1, 0], device="cuda")

    def plain(head, x):
        z = x.view(n, T, 6, F // 6)
        z = (z - z.mean(3, keepdim=True)) / torch.sqrt(z.var(3, unbiased=False, keepdim=True) + 1e-5)
        z = z.reshape(n, T, F) * head.weight + head.bias
        p = torch.nn.functional.linear(z * torch.sigmoid(z), head.project.weight, head.project.bias)
        v, f, o = p.split(D, dim=2)
        h, total = torch.zeros(n, D, dtype=x.dtype, device="cuda"), 0.0
        for t in range(T):
            on = (lengths > t)[:, None]
            a = torch.sigmoid(f[:, t])
            h = torch.where(on, a * h + (1 - a) * v[:, t], h)
            total = total + torch.where(on, torch.sigmoid(o[:, t]) * h + v[:, t], 0.0 * h)
        mean = total / lengths.clamp(min=1)[:, None]
        return torch.nn.functional.linear(mean, head.classify.weight, head.classify.bias)

    loss = torch.nn.functional.cross_entropy(head(x, lengths), labels)
    loss.backward()
    got = {k: t.grad.double() for k, t in head.named_parameters()}
    ref = window_head.Head(F, 6, D, 3, p=0.0).cuda()
    ref.load_state_dict(head.state_dict())
    ref = ref.double()
    want = torch.nn.functional.cross_entropy(plain(ref, x.double()), labels)
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) < 1e-5
    for k, t in ref.named_parameters():
        scale = float(t.grad.abs().max())
        # fp32 products of 60 and sums over 45 rows: about 1e-6 of the largest
        assert float((got[k] - t.grad).abs().max()) < 2e-5 * scale + 1e-7, k


def test_wrappers_take_gradients_of_any_strides():
    """A sum's gradient is one number for every element (strides of 0)."""
    import torch

    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import window_head
    finally:
        sys.path.pop(0)
    n, T, C = 3, 7, 12
    x, p, r = (torch.randn(n, T, c, device="cuda", requires_grad=True) for c in (C, 3 * C, C))
    w, b = (torch.randn(C, device="cuda", requires_grad=True) for _ in range(2))
    lengths = torch.tensor([7, 0, 3], dtype=torch.int32, device="cuda")
    for call, inputs in ((lambda: window_head.GroupNorm.apply(x, w, b, 4, "silu"), (x, w, b)),
                         (lambda: window_head.Recurrence.apply(p, lengths), (p,)),
                         (lambda: window_head.Dropout.apply(x, r, 0.5, 1, 2), (x, r))):
        got = torch.autograd.grad(call().sum(), inputs)
        want = torch.autograd.grad(call(), inputs, torch.ones(n, T, C, device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
