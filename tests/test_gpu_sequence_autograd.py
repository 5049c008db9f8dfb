"""What the sequence operators owe to torch's autograd, which they do not record
themselves for."""
import pytest

from test_gpu_sequence import env  # noqa: F401

pytestmark = pytest.mark.gpu


def calls(torch, seq):
    """(names of operands, a call of them) of every operator."""
    x, h, w = torch.randn(2, 6, 8, device="cuda"), torch.randn(2, 8, device="cuda"), torch.ones(8, device="cuda")
    m, states = torch.randn(2, 4, device="cuda"), torch.randn(2, 1, 8, device="cuda")
    return [
        (lambda x, w, b: seq.group_norm(x, 4, w, b), (x, w, w)),
        (lambda dy, x, m, r, w, b: seq.group_norm_backward(dy, x, 4, m, r, w, b), (x, x, m, m, w, w)),
        (lambda v, f, o, h0: seq.recurrence(v, f, o, h0=h0), (x, x, x, h)),
        (lambda dy, v, f, s, o, dl: seq.recurrence_backward(dy, v, f, s, o, dh_last=dl), (x, x, x, states, x, h)),
        (lambda v, f, h, o: seq.recurrence_step(v, f, h, o), (h, h, h, h)),
        (lambda x, r: seq.dropout(x, 0.5, 1, residual=r), (x, x)),
        (lambda dy: seq.dropout_backward(dy, 0.5, 1), (x,))]


def test_operands_that_require_gradients_are_refused(env):  # noqa: F811
    torch, seq = env
    for call, operands in calls(torch, seq):
        call(*operands)
        for k in range(len(operands)):
            wanting = [t.clone().requires_grad_(True) if i == k else t for i, t in enumerate(operands)]
            with pytest.raises(ValueError, match="requires gradients"):
                call(*wanting)
            with torch.no_grad():
                call(*wanting)


def test_outputs_that_require_gradients_are_refused(env):  # noqa: F811
    torch, seq = env
    x, h = torch.randn(2, 6, 8, device="cuda"), torch.randn(2, 8, device="cuda")
    leaf, leaf_h = x.clone().requires_grad_(True), h.clone().requires_grad_(True)
    m, states = torch.randn(2, 4, device="cuda"), torch.randn(2, 1, 8, device="cuda")
    for call in (lambda: seq.group_norm(x, 4, out=leaf), lambda: seq.group_norm_backward(x, x, 4, m, m, out=leaf),
                 lambda: seq.recurrence(x, x, out=leaf), lambda: seq.dropout(x, 0.5, 1, out=leaf),
                 lambda: seq.recurrence_backward(x, x, x, states, out=[x.clone(), leaf]),
                 lambda: seq.recurrence_step(h, h, h, out=leaf_h), lambda: seq.recurrence_step(h, h, h, h_out=leaf_h)):
        with pytest.raises(ValueError, match="requires gradients"):
            call()


def test_outputs_over_saved_tensors_are_noticed(env):  # noqa: F811
    """What autograd saved and a call wrote over is an error in the backward
    pass, as after torch's own operations in place."""
    torch, seq = env
    x, h = torch.randn(2, 6, 8, device="cuda"), torch.randn(2, 8, device="cuda")
    m, states = torch.randn(2, 4, device="cuda"), torch.randn(2, 1, 8, device="cuda")
    for like, call in ((x, lambda t: seq.group_norm(t, 4, out=t)), (x, lambda t: seq.recurrence(t, x, out=t)),
                       (x, lambda t: seq.group_norm_backward(t, x, 4, m, m, out=t)),
                       (x, lambda t: seq.recurrence_backward(x, x, x, states, out=[x.clone(), t])),
                       (h, lambda t: seq.recurrence_step(h, h, t, h_out=t)),
                       (h, lambda t: seq.recurrence_step(t, h, h, out=t)),
                       (x, lambda t: seq.dropout(t, 0.5, 1, out=t)),
                       (x, lambda t: seq.dropout_backward(t, 0.5, 1, out=t))):
        saved = like.clone()
        w = torch.ones_like(like, requires_grad=True)
        loss = (saved * w).sum()
        call(saved)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    with torch.inference_mode():   # such tensors keep no versions
        t = x.clone()
        seq.group_norm(t, 4, out=t)
