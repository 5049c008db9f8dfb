"""Timed cases of the operators around a trained head's linear layers: RMS norm with a residual, products in 8 bits
and 8-bit checkpoints.

The transform gives a feature row of hundreds to 20,000 features for every window, so a long series becomes a
sequence [n, L, C]: n series, L windows, C features, channels last.  A head normalises each row, projects it to N
channels, and in training keeps the rows for the projection's gradient.

The keys of a case:
  op       "norm", "norm_back", "norm_linear8", "linear8", "keep" or "weight_gradient"
  n, L, C  series, steps, channels
  dtype    type of the sequences that come in ("float32", "bfloat16", "float16"); weights, scales, statistics and
           weights' gradients are float32
  ragged   every series has a length of its own, from 0 to L; steps past it hold no data (they hold NaN here) and
           give zeros
  residual (norm, norm_back, norm_linear8) a residual is added first, and its sum is given (in the backward pass:
           a gradient of the sum comes in)
  N        (norm_linear8, linear8, weight_gradient) channels that the projection gives
  out      (norm_linear8, linear8, keep) type of the result

RMS norm of a row:
    s = x + residual, rounded to the type;  k = 1 / sqrt(mean of s^2 + eps);  y = s k w
Its rows in 8 bits, for a product:
    a = the largest |s w| of the row, q = s w 127 / a to the nearest whole number (ties to even), scale = k a / 127
Product in 8 bits, the channels padded with zeros to a multiple of 64:
    y = scale_row wscale_n (sum of q p_n) + b_n
Checkpoint, blocks of 128 rows (all series' steps in a row), a scale for each channel of a block:
    a = the largest |x| of the channel's 128 values, q = x 127 / a to the nearest whole number, scale = a / 127;
    restored q scale.  Kept as q [blocks, C, 128] and scale [blocks, C].
Weight gradient of y = x W^T + b from the checkpoint: dW = sum over rows of dy (q scale), db = sum of dy
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
BLOCK = 128             # rows that share a channel's scale in a checkpoint
PAD = 64                # columns of 8-bit rows come in multiples
LARGEST_BYTES = 2.1e9   # of the listed cases
LARGEST_FLOPS = 4e11
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _case(op, n, L, C, dtype, ragged=False, **more):
    return dict(op=op, n=n, L=L, C=C, dtype=dtype, ragged=ragged, **more)


def listed():
    return [
        # one window of a running service: the 2,000 features of 1,000 kernels, normalised and projected to the
        # three blocks of a recurrence of 64 channels
        dict(_case("norm_linear8", 1, 1, 2000, "float32", residual=False, N=192, out="bfloat16"),
             name="norm_linear8_step"),
        # between two blocks of a deep head, in training
        dict(_case("norm", 500, 1000, 256, "bfloat16", residual=True), name="norm_residual"),
        # the features of 10,000 kernels as the transform gives them
        dict(_case("norm", 2048, 1, 20000, "float32", residual=False), name="norm_wide"),
        # the same block's gradient over a production line's sequences
        dict(_case("norm_back", 1000, 1000, 256, "bfloat16", residual=True), name="norm_back"),
        # one new step for every stream of a service
        dict(_case("linear8", 64, 1, 2000, "int8", N=1536, out="bfloat16"), name="linear8_step"),
        # an ordinary batch of sequences: the most work
        dict(_case("linear8", 64, 1000, 2000, "int8", N=1536, out="bfloat16"), name="linear8_batch"),
        # series of unequal lengths, MINIROCKET's 924 features, an odd number of channels
        dict(_case("linear8", 777, 129, 924, "int8", ragged=True, N=993, out="float16"), name="linear8_ragged"),
        # features kept for the backward pass and read back in the type that trains
        dict(_case("keep", 64, 1000, 2000, "float32", out="bfloat16"), name="keep"),
        # an odd number of channels, series of unequal lengths
        dict(_case("keep", 777, 129, 331, "float16", ragged=True, out="float16"), name="keep_ragged"),
        # the projection's gradient in an ordinary training step
        dict(_case("weight_gradient", 64, 1000, 2000, "bfloat16", N=1536), name="weight_gradient"),
        # the same of ragged series and odd sizes
        dict(_case("weight_gradient", 777, 129, 924, "float16", ragged=True, N=993), name="weight_gradient_ragged"),
        # a small study's batch in full precision
        dict(_case("weight_gradient", 64, 1, 2000, "float32", N=192), name="weight_gradient_small"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    while True:
        op = rng.choice(["norm", "norm", "norm_back", "norm_back", "norm_linear8", "linear8", "linear8", "linear8",
                         "keep", "keep", "weight_gradient", "weight_gradient", "weight_gradient"])
        dtype, out = rng.choice(sorted(TYPES)), rng.choice(sorted(TYPES))
        n, L, C, N = log_int(1, 1000), log_int(1, 20000), log_int(8, 20000), log_int(2, 2000)
        if rng.random() < 0.5:
            C = max(8, C // 8 * 8)
        if rng.random() < 0.2:   # a step of every stream
            L = 1
        ragged = L > 1 and rng.random() < 0.3
        if op in ("norm", "norm_back"):
            case = _case(op, n, L, C, dtype, ragged, residual=rng.random() < 0.5)
        elif op == "norm_linear8":
            case = _case(op, n, L, C, dtype, ragged, residual=rng.random() < 0.5, N=N,
                         out=rng.choice(["bfloat16", "float16"]))
        elif op == "linear8":
            case = _case(op, n, L, C, "int8", ragged, N=N, out=out)
        elif op == "keep":
            case = _case(op, n, L, C, dtype, ragged, out=rng.choice(["bfloat16", "float16"]))
        else:
            case = _case(op, n, L, C, dtype, ragged, N=N)
        w = work(case)
        if w["bytes"] <= LARGEST_BYTES and w["flops"] <= LARGEST_FLOPS and n * L * C <= 2.6e8:
            return case


# ------------------------------------------------------------------ inputs
def _lengths(case, gen):
    """None, or int32 [n] on the GPU: 0 to L, and the whole L for one series at least."""
    if not case["ragged"]:
        return None
    t = torch.randint(0, case["L"] + 1, (case["n"],), generator=gen, device="cuda", dtype=torch.int32)
    t[0] = case["L"]
    return t


def _past(n, L, lengths, device):
    return torch.arange(L, device=device)[None, :] >= lengths[:, None]


def _blank(x, lengths):
    """x with NaN at the steps past each series' length."""
    if lengths is not None:
        x.masked_fill_(_past(x.shape[0], x.shape[1], lengths, x.device)[:, :, None], float("nan"))
    return x


def _padded(C):
    return -(-C // PAD) * PAD


def _weight_rows(w):
    """8-bit rows of a weight matrix [N, C] and their scales, padded: made once, when the model is loaded."""
    top = w.abs().amax(1, keepdim=True)
    q = torch.zeros((w.shape[0], _padded(w.shape[1])), dtype=torch.int8, device=w.device)
    q[:, :w.shape[1]] = torch.round(w * (127.0 / top))
    return q, (top / 127.0).view(-1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, L, C, op = case["n"], case["L"], case["C"], case["op"]
    dt = TYPES.get(case["dtype"])

    def normal(*shape, scale=1.0, shift=0.0, dtype=torch.float32):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = dict(case=case, lengths=_lengths(case, gen))
    lengths = s["lengths"]
    # features differ in level and spread from channel to channel
    level, spread = normal(C), normal(C, scale=0.3).exp()

    def features():
        return torch.randn((n, L, C), generator=gen, device="cuda").mul_(spread).add_(level)

    if op in ("norm", "norm_back", "norm_linear8"):
        s.update(x=_blank(features().to(dt), lengths), weight=normal(C, scale=0.2, shift=1.0), residual=None)
        if op == "norm_back":   # x is the sum that the forward pass gave
            s.update(rstd=_rstd(s["x"], lengths), dy=_blank(normal(n, L, C, dtype=dt), lengths),
                     dtotal=_blank(normal(n, L, C, dtype=dt), lengths) if case["residual"] else None)
        elif case["residual"]:
            s.update(residual=_blank(normal(n, L, C, scale=2.0, dtype=dt), lengths))
    if op in ("norm_linear8", "linear8"):
        N = case["N"]
        wq, wscale = _weight_rows(normal(N, C, scale=C ** -0.5))
        s.update(wq=wq, wscale=wscale, bias=normal(N, scale=0.1), out=TYPES[case["out"]])
    if op == "linear8":
        # rows as the norm gives them: their largest value is 127
        q = torch.zeros((n, L, _padded(C)), dtype=torch.int8, device="cuda")
        q[:, :, :C] = torch.randn((n, L, C), generator=gen, device="cuda").mul_(36.0).round_().clamp_(-127, 127)
        q[:, :, 0] = 127
        scale = torch.rand((n, L), generator=gen, device="cuda").mul_(0.02).add_(0.02)
        if lengths is not None:
            scale.masked_fill_(_past(n, L, lengths, scale.device), float("nan"))
        s.update(q=q, scale=scale)
    elif op == "keep":
        s.update(x=_blank(features().to(dt), lengths), out=TYPES[case["out"]])
    elif op == "weight_gradient":
        blocks = -(-n * L // BLOCK)
        q = torch.randint(-127, 128, (blocks, C, BLOCK), generator=gen, device="cuda", dtype=torch.int8)
        dead = torch.zeros(blocks * BLOCK, dtype=torch.bool, device="cuda")   # rows that hold no data are zeros
        dead[n * L:] = True
        if lengths is not None:
            dead[:n * L] = _past(n, L, lengths, q.device).view(-1)
        q.masked_fill_(dead.view(blocks, 1, BLOCK), 0)
        scale = torch.rand((blocks, C), generator=gen, device="cuda").mul_(0.5).add_(0.75).mul_(spread / 40)
        s.update(q=q, scale=scale, dy=_blank(normal(n, L, case["N"], scale=0.01).to(dt), lengths))
    return s


# -------------------------------------------------------------- plain forms
def _own_steps(x, lengths):
    """x in float32, 0 at the steps past each series' length."""
    x = x.float()
    if lengths is None:
        return x
    return x.masked_fill(_past(x.shape[0], x.shape[1], lengths, x.device)[:, :, None], 0.0)


def _own_rows(v, lengths):
    """The same for one value a step, [n, L]."""
    return v if lengths is None else v.masked_fill(_past(v.shape[0], v.shape[1], lengths, v.device), 0.0)


def _rstd(total, lengths):
    f = _own_steps(total, lengths)
    return _own_rows(1.0 / torch.sqrt((f * f).mean(2) + EPS), lengths)


def _total(s):
    """The sum that is normalised, rounded to the type; without a residual it is x."""
    if s["residual"] is None:
        return s["x"]
    return _own_steps(s["x"].float() + s["residual"].float(), s["lengths"]).to(s["x"].dtype)


def _plain_norm(s):
    total = _total(s)
    rstd = _rstd(total, s["lengths"])
    y = _own_steps(total, s["lengths"]) * rstd[:, :, None] * s["weight"]
    out = dict(y=y.to(total.dtype), rstd=rstd)
    return out if s["residual"] is None else dict(out, total=total)


def _plain_norm_back(s):
    f, r = _own_steps(s["x"], s["lengths"]), s["rstd"][:, :, None]
    dy = _own_steps(s["dy"], s["lengths"])
    g = dy * s["weight"]
    xh = f * r
    dx = r * (g - xh * (g * xh).mean(2, keepdim=True))
    if s["dtotal"] is not None:
        dx = dx + _own_steps(s["dtotal"], s["lengths"])
    return dict(dx=dx.to(s["x"].dtype), dweight=(dy * xh).sum(dim=(0, 1)))


def _plain_product(q, scale, s):
    y = (q.float() @ s["wq"].float().t()) * scale[:, :, None] * s["wscale"] + s["bias"]
    return _own_steps(y, s["lengths"]).to(s["out"])


def _plain_linear8(s):
    return _plain_product(s["q"], _own_rows(s["scale"], s["lengths"]), s)


def _plain_norm_linear8(s):
    total = _total(s)
    rstd = _rstd(total, s["lengths"])
    v = _own_steps(total, s["lengths"]) * s["weight"]
    top = v.abs().amax(2)
    inverse = torch.where(top > 0, 127.0 / top, torch.zeros_like(top))
    q = torch.round(v * inverse[:, :, None])
    q = torch.nn.functional.pad(q, (0, _padded(q.shape[2]) - q.shape[2]))
    out = dict(y=_plain_product(q, rstd * top / 127.0, s), rstd=rstd)
    return out if s["residual"] is None else dict(out, total=total)


def _plain_keep(s):
    f = _own_steps(s["x"], s["lengths"])
    n, L, C = f.shape
    f = torch.nn.functional.pad(f.view(n * L, C), (0, 0, 0, -n * L % BLOCK)).view(-1, BLOCK, C)
    top = f.abs().amax(1, keepdim=True)
    q = torch.round(f * torch.where(top > 0, 127.0 / top, torch.zeros_like(top))).to(torch.int8)
    scale = top / 127.0
    x = (q.float() * scale).view(-1, C)[:n * L].view(n, L, C)
    return dict(x=x.to(s["out"]), scale=scale.view(-1, C))


def _plain_weight_gradient(s):
    dy = _own_steps(s["dy"], s["lengths"])
    n, L, N = dy.shape
    dy = dy.view(n * L, N)
    x = (s["q"].float() * s["scale"][:, :, None]).transpose(1, 2).reshape(-1, s["q"].shape[1])[:n * L]
    return dict(dweight=dy.t() @ x, dbias=dy.sum(0))


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return dict(norm=_plain_norm, norm_back=_plain_norm_back, norm_linear8=_plain_norm_linear8,
                    linear8=_plain_linear8, keep=_plain_keep, weight_gradient=_plain_weight_gradient)[op](s)
    from paper_2601_17091_amd import sequence
    if op == "norm":
        y, total, rstd = sequence.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, lengths=s["lengths"])
        return dict(y=y, rstd=rstd) if s["residual"] is None else dict(y=y, rstd=rstd, total=total)
    if op == "norm_back":
        dx, dweight = sequence.rms_norm_backward(s["dy"], s["x"], s["rstd"], s["weight"], dtotal=s["dtotal"],
                                                 lengths=s["lengths"])
        return dict(dx=dx, dweight=dweight)
    if op == "norm_linear8":
        q, scale, total, rstd = sequence.rms_norm8(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                                                   lengths=s["lengths"])
        y = sequence.linear8(q, scale, s["wq"], s["wscale"], s["bias"], dtype=s["out"], lengths=s["lengths"])
        return dict(y=y, rstd=rstd) if s["residual"] is None else dict(y=y, rstd=rstd, total=total)
    if op == "linear8":
        return sequence.linear8(s["q"], s["scale"], s["wq"], s["wscale"], s["bias"], dtype=s["out"],
                                lengths=s["lengths"])
    if op == "keep":
        q, scale = sequence.checkpoint(s["x"], lengths=s["lengths"])
        x = sequence.restore(q, scale, s["x"].shape[:2], dtype=s["out"], lengths=s["lengths"])
        return dict(x=x, scale=scale)
    dweight, dbias = sequence.linear_weight_gradient(s["dy"], s["q"], s["scale"], lengths=s["lengths"])
    return dict(dweight=dweight, dbias=dbias)


# ------------------------------------------------------------------- floors
def work(case):
    """Bytes: each input read once, each output written once; of ragged inputs the half that random lengths hold on
    average (outputs are whole: the rest of them is zeros).  A checkpoint is written and read again.  flops: a
    multiplication and an addition of a product are two."""
    n, L, C, op, N = case["n"], case["L"], case["C"], case["op"], case.get("N", 0)
    size = {"float32": 4, "int8": 1}.get(case["dtype"], 2)
    out = {"float32": 4, None: 0}.get(case.get("out"), 2)
    rows = n * L
    live = rows / 2 if case["ragged"] else rows
    both = 2 if case.get("residual") else 1
    if op == "norm":
        need, flops = both * (live + rows) * C * size + 4 * rows + 4 * C, 6 * live * C
    elif op == "norm_back":
        need, flops = ((1 + both) * live + rows) * C * size + 4 * rows + 8 * C, 11 * live * C
    elif op == "norm_linear8":
        need = (both * live + (both - 1) * rows) * C * size + 4 * rows + rows * N * out + N * C + 4 * C + 8 * N
        flops = 2 * live * C * N + 6 * live * C
    elif op == "linear8":
        need, flops = live * C + 4 * live + rows * N * out + N * C + 8 * N, 2 * live * C * N
    elif op == "keep":
        need = live * C * size + 2 * rows * C + 3 * 4 * C * (rows / BLOCK) + rows * C * out
        flops = 4 * live * C
    else:
        need = live * N * size + rows * C + 4 * C * (rows / BLOCK) + 4 * N * C + 4 * N
        flops = 2 * live * C * N
    return dict(bytes=int(need), flops=int(flops))


# --------------------------------------------------- the definitions, 64 bits
def _live(s, n, L, device):
    """[n, L, 1] of 1 and 0 in 64 bits."""
    if s["lengths"] is None:
        return torch.ones((n, L, 1), dtype=torch.float64, device=device)
    steps = torch.arange(L, device=device).expand(n, L)
    return (steps < s["lengths"].view(n, 1)).double().unsqueeze(2)


def _held(t, live):
    """t in 64 bits with zeros where nothing is live (NaN there included)."""
    return torch.where(live > 0, t.double(), torch.zeros((), dtype=torch.float64, device=t.device))


def _exact_rows(s):
    """live, the sum as it is kept (of the type), its values, rstd."""
    x = s["x"]
    live = _live(s, x.shape[0], x.shape[1], x.device)
    kept = x
    if s["residual"] is not None:
        kept = _held((x.double() + s["residual"].double()).to(x.dtype), live)
    v = _held(kept, live)
    rstd = (v.square().sum(2, keepdim=True) / v.shape[2] + EPS).rsqrt() * live
    return live, kept, v, rstd


def _exact_norm(s):
    live, kept, v, rstd = _exact_rows(s)
    out = dict(y=s["weight"].double() * (v * rstd), rstd=rstd.squeeze(2))
    return out if s["residual"] is None else dict(out, total=kept)


def _exact_norm_back(s):
    x = s["x"]
    live = _live(s, x.shape[0], x.shape[1], x.device)
    v, dy, k = _held(x, live), _held(s["dy"], live), s["rstd"].double().unsqueeze(2)
    g = dy * s["weight"].double()
    inner = (g * v).sum(2, keepdim=True) / v.shape[2]
    dx = k * g - v * inner * k ** 3
    if s["dtotal"] is not None:
        dx += _held(s["dtotal"], live)
    return dict(dx=dx, dweight=(dy * v * k).sum(dim=(0, 1)))


def _exact_product(q, scale, s, live):
    N = s["wq"].shape[0]
    rows = torch.empty(q.shape[:2] + (N,), dtype=torch.float64, device=q.device)
    w = s["wq"].double().mul(s["wscale"].double().unsqueeze(1)).t().contiguous()
    flat, to = q.view(-1, q.shape[2]), rows.view(-1, N)
    for at in range(0, flat.shape[0], 1 << 16):
        torch.mm(flat[at:at + (1 << 16)].double(), w, out=to[at:at + (1 << 16)])
    return _held((rows * scale.double().unsqueeze(2) + s["bias"].double()), live)


def _exact_linear8(s):
    live = _live(s, s["q"].shape[0], s["q"].shape[1], s["q"].device)
    return _exact_product(s["q"], s["scale"], s, live)


def _exact_norm_linear8(s):
    live, kept, v, rstd = _exact_rows(s)
    v = v * s["weight"].double()
    top = v.abs().max(2).values
    unit = (top / 127).clamp(min=1e-300).unsqueeze(2)
    q = torch.zeros(v.shape[:2] + (s["wq"].shape[1],), dtype=torch.float64, device=v.device)
    q[:, :, :v.shape[2]] = (v / unit).round()
    out = dict(y=_exact_product(q, rstd.squeeze(2) * top / 127, s, live), rstd=rstd.squeeze(2))
    return out if s["residual"] is None else dict(out, total=kept)


def _exact_keep(s):
    x = s["x"]
    n, L, C = x.shape
    v = _held(x, _live(s, n, L, x.device)).view(n * L, C)
    scales = torch.empty((-(-n * L // BLOCK), C), dtype=torch.float64, device=x.device)
    for b in range(scales.shape[0]):
        part = v[b * BLOCK:(b + 1) * BLOCK]
        scales[b] = part.abs().max(0).values / 127
        unit = scales[b].clamp(min=1e-300)
        part.copy_((part / unit).round() * unit)
    return dict(x=v.view(n, L, C), scale=scales)


def _exact_weight_gradient(s):
    dy, q = s["dy"], s["q"]
    n, L, N = dy.shape
    dy = _held(dy, _live(s, n, L, dy.device)).view(n * L, N)
    dweight = torch.zeros((N, q.shape[1]), dtype=torch.float64, device=dy.device)
    step = 256   # blocks
    for at in range(0, q.shape[0], step):
        part = dy[at * BLOCK:(at + step) * BLOCK]
        x = q[at:at + step].permute(0, 2, 1) * s["scale"][at:at + step].double().unsqueeze(1)
        dweight.addmm_(part.t(), x.reshape(-1, q.shape[1])[:part.shape[0]])
    return dict(dweight=dweight, dbias=dy.sum(0))


def exact(case, seed):
    s = prepare(case, seed)
    return dict(norm=_exact_norm, norm_back=_exact_norm_back, norm_linear8=_exact_norm_linear8,
                linear8=_exact_linear8, keep=_exact_keep, weight_gradient=_exact_weight_gradient)[case["op"]](s)
