"""Timed cases of the sequence operators: what a trained head over ROCKET features runs.

The transform gives a feature row for every window of a series, so a long
series becomes a sequence [n, L, C]: n series, L windows (or samples), C
channels, channels last.  A learned head over such sequences normalises the
features by groups with an activation, mixes them over time with a gated
linear recurrence and regularises with dropout.

The keys of a case:
  op       "norm", "norm_back", "rec", "rec_step", "rec_back", "drop" or
           "drop_back"
  n, L, C  series, steps, channels
  dtype    type of the sequences ("float32", "bfloat16", "float16");
           statistics, weights, states and their gradients are float32
  ragged   every series has a length of its own, from 0 to L; steps past it
           hold no data (they hold NaN here) and give zeros
  norm:    groups, act ("none", "relu", "silu", "gelu")
  rec:     gate (the output gate is there), packed (v, f and o are column
           blocks of one projection's output [n, L, 2C or 3C]), state (an
           initial state comes in, and in the backward pass a gradient of the
           last state), keep (a forward pass in training, which also returns
           the states before the steps 0, 128, 256, ... for the backward pass)
  drop:    p, residual (y = residual + dropout(x)), call (the call's number,
           which may pass 32 bits)

Group norm over a series of T steps, group g of C / groups channels:
    m = mean of x over the T steps and the group's channels, s = the mean of
    (x - m)^2 there, r = 1 / sqrt(s + eps)
    z = (x - m) r w_c + b_c,   y = act(z);   m = r = 0 where T = 0
Recurrence, with S the logistic function:
    h_t = S(f_t) h_{t-1} + (1 - S(f_t)) v_t,   y_t = S(o_t) h_t or h_t;
    steps past a series' length leave h as it is
Dropout: Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011) with the key
(seed low, seed high) and the counter (i / 8 low, i / 8 high, call low, call
high) gives eight 16-bit numbers for the elements 8 (i / 8) + 0..7, low halves
before high halves, word by word; an element is dropped where its number is
below D = round(65536 p), and kept ones are scaled by 65536 / (65536 - D).
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
EVERY = 128        # steps between the states that training keeps
LARGEST = 1.54e9   # bytes of the largest listed case
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _norm(op, n, L, C, groups, dtype, act, ragged=False):
    return dict(op=op, n=n, L=L, C=C, groups=groups, dtype=dtype, act=act, ragged=ragged)


def _rec(op, n, L, C, dtype, gate, packed=False, state=False, ragged=False, keep=False):
    return dict(op=op, n=n, L=L, C=C, dtype=dtype, gate=gate, packed=packed, state=state, ragged=ragged, keep=keep)


def _drop(op, n, L, C, dtype, p, residual=False, call=0):
    return dict(op=op, n=n, L=L, C=C, dtype=dtype, p=p, residual=residual, call=call)


def listed():
    return [
        # one window of a running service: the 2,000 features of 1,000 kernels
        dict(_norm("norm", 1, 1, 2000, 20, "float32", "none"), name="norm_one_window"),
        # series of unequal lengths, MINIROCKET's 924 features in groups of 33
        dict(_norm("norm", 777, 129, 924, 28, "float16", "relu", ragged=True), name="norm_ragged"),
        # few long recordings: one group's slab is far larger than a workgroup holds
        dict(_norm("norm", 4, 16384, 512, 8, "bfloat16", "gelu"), name="norm_few_long"),
        # a training step over a production line's sequences: the largest case
        dict(_norm("norm_back", 1000, 1000, 256, 16, "bfloat16", "silu"), name="norm_back"),
        # one new step for every stream of a service
        dict(_rec("rec_step", 64, 1, 512, "bfloat16", gate=True, packed=True, state=True), name="rec_step"),
        # ragged series through an odd number of channels, in training
        dict(_rec("rec", 777, 129, 331, "float16", gate=True, ragged=True, keep=True), name="rec_ragged"),
        # few long recordings: the time axis is all there is to split
        dict(_rec("rec", 4, 16384, 256, "bfloat16", gate=False, state=True), name="rec_few_long"),
        # an ordinary training batch, the gates from one projection
        dict(_rec("rec_back", 64, 1000, 512, "bfloat16", gate=True, packed=True), name="rec_back"),
        # training on long recordings in full precision
        dict(_rec("rec_back", 8, 10000, 256, "float32", gate=False, state=True), name="rec_back_long"),
        # regularised features of a small study's batch
        dict(_drop("drop", 64, 1, 2000, "float32", 0.5), name="drop_small"),
        # the residual join after a block, in training
        dict(_drop("drop", 500, 1000, 256, "bfloat16", 0.1, residual=True, call=12345), name="drop_residual"),
        # gradient of an odd number of elements, late in a long run
        dict(_drop("drop_back", 777, 129, 331, "float16", 0.25, call=(1 << 33) + 7), name="drop_back"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    while True:
        op = rng.choice(["norm", "norm", "norm_back", "norm_back", "rec", "rec", "rec_step", "rec_back",
                         "rec_back", "drop", "drop_back"])
        dtype = rng.choice(sorted(TYPES))
        n, L = log_int(1, 1000), log_int(1, 20000)
        C = log_int(8, 2000)
        if rng.random() < 0.5:
            C = max(8, C // 8 * 8)
        ragged = rng.random() < 0.3
        if op in ("norm", "norm_back"):
            width = log_int(1, C)
            groups = max(g for g in range(1, C + 1) if C % g == 0 and g <= max(1, C // width))
            case = _norm(op, n, L, C, groups, dtype, rng.choice(["none", "relu", "silu", "gelu"]), ragged)
        elif op == "rec_step":
            case = _rec(op, log_int(1, 4000), 1, C, dtype, rng.random() < 0.5, rng.random() < 0.5, True)
        elif op in ("rec", "rec_back"):
            case = _rec(op, n, L, C, dtype, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5, ragged,
                        op == "rec" and rng.random() < 0.5)
        else:
            case = _drop(op, n, L, C, dtype, round(rng.uniform(0.01, 0.9), 4),
                         op == "drop" and rng.random() < 0.5, rng.randrange(1 << 36))
        if work(case)["bytes"] <= LARGEST:
            return case


# ------------------------------------------------------------------ inputs
def _lengths(case, gen):
    """None, or int32 [n] on the GPU: 0 to L, and the whole L for one series at least."""
    if not case.get("ragged"):
        return None
    t = torch.randint(0, case["L"] + 1, (case["n"],), generator=gen, device="cuda", dtype=torch.int32)
    t[0] = case["L"]
    return t


def _blank(x, lengths):
    """x with NaN at the steps past each series' length."""
    if lengths is not None:
        past = torch.arange(x.shape[1], device=x.device)[None, :] >= lengths[:, None]
        x.masked_fill_(past[:, :, None], float("nan"))
    return x


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, L, C, dt, op = case["n"], case["L"], case["C"], TYPES[case["dtype"]], case["op"]

    def normal(*shape, scale=1.0, shift=0.0, dtype=dt):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = dict(case=case, lengths=_lengths(case, gen))
    if op in ("norm", "norm_back"):
        # features differ in level and spread from channel to channel
        level, spread = normal(C, dtype=torch.float32), normal(C, scale=0.3, dtype=torch.float32).exp()
        x = torch.randn((n, L, C), generator=gen, device="cuda").mul_(spread).add_(level).to(dt)
        s.update(x=_blank(x, s["lengths"]),
                 weight=normal(C, scale=0.2, shift=1.0, dtype=torch.float32),
                 bias=normal(C, scale=0.2, dtype=torch.float32))
        if op == "norm_back":
            # the statistics that the forward pass kept
            mean, rstd = _statistics(x, case["groups"], s["lengths"])
            s.update(dy=_blank(normal(n, L, C), s["lengths"]), mean=mean, rstd=rstd)
    elif op == "rec_step":
        parts = 3 if case["gate"] else 2
        if case["packed"]:
            p = normal(n, parts * C)
            s.update(v=p[:, :C], f=p[:, C:2 * C].add_(1.0), o=p[:, 2 * C:] if case["gate"] else None)
        else:
            s.update(v=normal(n, C), f=normal(n, C, shift=1.0), o=normal(n, C) if case["gate"] else None)
        s.update(h=normal(n, C, scale=0.5, dtype=torch.float32))
    elif op in ("rec", "rec_back"):
        parts = 3 if case["gate"] else 2
        # gates that mostly keep: memories of a few steps to hundreds of them
        shift = torch.linspace(0.0, 5.0, C, device="cuda")
        if case["packed"]:
            p = torch.randn((n, L, parts * C), generator=gen, device="cuda")
            p[:, :, C:2 * C] += shift
            p = _blank(p, s["lengths"]).to(dt)
            v, f, o = p[:, :, :C], p[:, :, C:2 * C], p[:, :, 2 * C:] if case["gate"] else None
        else:
            v = _blank(normal(n, L, C), s["lengths"])
            f = _blank(torch.randn((n, L, C), generator=gen, device="cuda").add_(shift), s["lengths"]).to(dt)
            o = _blank(normal(n, L, C), s["lengths"]) if case["gate"] else None
        s.update(v=v, f=f, o=o, h0=normal(n, C, dtype=torch.float32) if case["state"] else None)
        if op == "rec_back":
            # the states that the forward pass kept
            s.update(states=_plain_rec(dict(s, case=dict(case, keep=True)))["states"])
            s.update(dy=_blank(normal(n, L, C), s["lengths"]),
                     dh_last=normal(n, C, dtype=torch.float32) if case["state"] else None, out=None)
            if case["packed"]:   # the gradients go where the projection's gradient is wanted
                d = torch.empty((n, L, parts * C), dtype=dt, device="cuda")
                s.update(out=[d[:, :, k * C:(k + 1) * C] for k in range(parts)])
    else:
        s.update(x=normal(n, L, C), seed=seed * 0x9E3779B97F4A7C15 % (1 << 64),
                 residual=normal(n, L, C) if case["residual"] else None)
    return s


# -------------------------------------------------------------- plain forms
def _rows(lengths, L, like):
    """1 at a series' own steps, 0 past them, [n, L, 1]; None where all are its own."""
    if lengths is None:
        return None
    return (torch.arange(L, device=like.device)[None, :] < lengths[:, None])[:, :, None]


def _own_steps(x, live):
    x = x.float()
    return x if live is None else torch.where(live, x, torch.zeros((), device=x.device))


def _count(case_n, L, C, groups, lengths, device):
    steps = torch.full((case_n,), L, device=device) if lengths is None else lengths
    return (steps.float() * (C // groups)).clamp(min=1.0)[:, None]


def _statistics(x, groups, lengths):
    """mean and rstd, float32 [n, groups]; 0 and 0 for a series of no steps."""
    n, L, C = x.shape
    live = _rows(lengths, L, x)
    count = _count(n, L, C, groups, lengths, x.device)
    xf = _own_steps(x, live).view(n, L, groups, C // groups)
    mean = xf.sum(dim=(1, 3)) / count
    d = xf - mean[:, None, :, None]
    if live is not None:
        d = d * live[..., None]
    rstd = 1.0 / torch.sqrt((d * d).sum(dim=(1, 3)) / count + EPS)
    if lengths is not None:
        rstd = rstd * (lengths > 0)[:, None]
    return mean, rstd


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros((), device=z.device, dtype=z.dtype))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def _plain_norm(s):
    x, G = s["x"], s["case"]["groups"]
    n, L, C = x.shape
    live = _rows(s["lengths"], L, x)
    mean, rstd = _statistics(x, G, s["lengths"])
    xh = (_own_steps(x, live).view(n, L, G, C // G) - mean[:, None, :, None]) * rstd[:, None, :, None]
    y = _act(xh.view(n, L, C) * s["weight"] + s["bias"], s["case"]["act"])
    return dict(y=_own_steps(y, live).to(x.dtype), mean=mean, rstd=rstd)


def _plain_norm_back(s):
    x, G = s["x"], s["case"]["groups"]
    n, L, C = x.shape
    live = _rows(s["lengths"], L, x)
    r = s["rstd"][:, None, :, None]
    xh = ((_own_steps(x, live).view(n, L, G, C // G) - s["mean"][:, None, :, None]) * r).view(n, L, C)
    dz = _own_steps(s["dy"], live) * _act_slope(xh * s["weight"] + s["bias"], s["case"]["act"])
    dweight, dbias = (dz * xh).sum(dim=(0, 1)), dz.sum(dim=(0, 1))
    g = (dz * s["weight"]).view(n, L, G, C // G)
    xh = xh.view(n, L, G, C // G)
    count = _count(n, L, C, G, s["lengths"], x.device)
    mg = (g.sum(dim=(1, 3)) / count)[:, None, :, None]
    mgx = ((g * xh).sum(dim=(1, 3)) / count)[:, None, :, None]
    dx = (r * (g - mg - xh * mgx)).view(n, L, C)
    return dict(dx=_own_steps(dx, live).to(x.dtype), dweight=dweight, dbias=dbias)


def _shift_scan(a, b):
    """h with h_t = a_t h_{t-1} + b_t along dim 1 from h = 0, by doubling the span that each step covers."""
    a, b = a.clone(), b.clone()
    span = 1
    while span < a.shape[1]:
        nb = b[:, span:] + a[:, span:] * b[:, :-span]
        na = a[:, span:] * a[:, :-span]
        b[:, span:], a[:, span:] = nb, na
        span *= 2
    return b


def _gates(s):
    """a = S(f) and 1 - a in float32, 1 and 0 past a series' length; v and S(o) there 0."""
    live = _rows(s["lengths"], s["v"].shape[1], s["v"])
    f = _own_steps(s["f"], live)
    a, keep = 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(f))
    if live is not None:
        a, keep = torch.where(live, a, torch.ones_like(a)), keep * live
    v = _own_steps(s["v"], live)
    so = None if s["o"] is None else 1 / (1 + torch.exp(-_own_steps(s["o"], live)))
    return live, a, keep, v, so


def _plain_states(a, b, h0):
    if h0 is not None:
        b = b.clone()
        b[:, 0] += a[:, 0] * h0
    return _shift_scan(a, b)


def _plain_rec(s):
    live, a, keep, v, so = _gates(s)
    h = _plain_states(a, keep * v, s["h0"])
    y = h if so is None else h * so
    out = dict(y=_own_steps(y, live).to(s["v"].dtype), h_last=h[:, -1].clone())
    if s["case"]["keep"]:
        first = torch.zeros_like(h[:, :1]) if s["h0"] is None else s["h0"][:, None]
        out["states"] = torch.cat([first, h[:, EVERY - 1:-1:EVERY]], dim=1)
    return out


def _plain_rec_back(s):
    live, a, keep, v, so = _gates(s)
    dt = s["v"].dtype
    h = _plain_states(a, keep * v, s["h0"])
    before = torch.empty_like(h)
    before[:, 1:] = h[:, :-1]
    before[:, 0] = 0 if s["h0"] is None else s["h0"]
    dy = _own_steps(s["dy"], live)
    g = dy if so is None else dy * so
    if s["dh_last"] is not None:
        g = g.clone()
        g[:, -1] += s["dh_last"]
    # dh_t = g_t + a_{t+1} dh_{t+1}: the same recurrence from the other end
    nxt = torch.zeros_like(a)
    nxt[:, :-1] = a[:, 1:]
    dh = _shift_scan(nxt.flip(1), g.flip(1)).flip(1)
    grads = [dh * keep, dh * (before - v) * a * keep]
    if so is not None:
        grads.append(dy * h * so * (1 - so))
    grads = [_own_steps(t, live).to(dt) for t in grads]
    if s["out"] is not None:
        grads = [o.copy_(t) for o, t in zip(s["out"], grads)]
    out = dict(dv=grads[0], df=grads[1], dh0=a[:, 0] * dh[:, 0])
    if so is not None:
        out["do"] = grads[2]
    return out


def _plain_rec_step(s):
    f = s["f"].float()
    h = s["h"] / (1 + torch.exp(-f)) + s["v"].float() / (1 + torch.exp(f))
    y = h if s["o"] is None else h / (1 + torch.exp(-s["o"].float()))
    return dict(y=y.to(s["v"].dtype), h=h)


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


LOW = 0xFFFFFFFF


def _plain_kept(n_elements, seed, call, p, device):
    """Whether each element stays, bool [n_elements]."""
    blocks = torch.arange((n_elements + 7) // 8, device=device)
    c = [blocks & LOW, blocks >> 32, torch.full_like(blocks, call & LOW), torch.full_like(blocks, call >> 32)]
    k0, k1 = seed & LOW, seed >> 32
    for _ in range(10):
        m0, m1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57   # wrapped products: their 64 bits are right
        c = [((m1 >> 32) & LOW) ^ c[1] ^ k0, m1 & LOW, ((m0 >> 32) & LOW) ^ c[3] ^ k1, m0 & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    halves = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], dim=1)
    return (halves >= _threshold(p)).view(-1)[:n_elements]


def _plain_drop(s):
    case, x = s["case"], s["x"]
    d = _threshold(case["p"])
    kept = _plain_kept(x.numel(), s["seed"], case["call"], case["p"], x.device).view(x.shape)
    y = torch.where(kept, x.float() * (65536.0 / max(1, 65536 - d)), torch.zeros((), device=x.device))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return dict(norm=_plain_norm, norm_back=_plain_norm_back, rec=_plain_rec, rec_back=_plain_rec_back,
                    rec_step=_plain_rec_step, drop=_plain_drop, drop_back=_plain_drop)[op](s)
    from paper_2601_17091_amd import sequence
    if op == "norm":
        y, mean, rstd = sequence.group_norm(s["x"], case["groups"], s["weight"], s["bias"], eps=EPS,
                                            activation=case["act"], lengths=s["lengths"])
        return dict(y=y, mean=mean, rstd=rstd)
    if op == "norm_back":
        dx, dweight, dbias = sequence.group_norm_backward(
            s["dy"], s["x"], case["groups"], s["mean"], s["rstd"], s["weight"], s["bias"],
            activation=case["act"], lengths=s["lengths"])
        return dict(dx=dx, dweight=dweight, dbias=dbias)
    if op == "rec":
        y, h_last, states = sequence.recurrence(s["v"], s["f"], s["o"], h0=s["h0"], lengths=s["lengths"],
                                                keep_states=case["keep"])
        return dict(y=y, h_last=h_last, states=states) if case["keep"] else dict(y=y, h_last=h_last)
    if op == "rec_back":
        dv, df, do, dh0 = sequence.recurrence_backward(s["dy"], s["v"], s["f"], s["states"], s["o"],
                                                       dh_last=s["dh_last"], lengths=s["lengths"], out=s["out"])
        out = dict(dv=dv, df=df, dh0=dh0)
        return out if do is None else dict(out, do=do)
    if op == "rec_step":
        y, h = sequence.recurrence_step(s["v"], s["f"], s["h"], s["o"])
        return dict(y=y, h=h)
    if op == "drop":
        return sequence.dropout(s["x"], case["p"], s["seed"], case["call"], residual=s["residual"])
    return sequence.dropout_backward(s["x"], case["p"], s["seed"], case["call"])


# ------------------------------------------------------------------- floors
def work(case):
    """Bytes: each input read once, each output written once; of ragged inputs
    the half that random lengths hold on average (outputs are whole: the rest
    of them is zeros).  flops: operations of the formulas, a transcendental
    counted as one, a Philox block as 100."""
    n, L, C, op = case["n"], case["L"], case["C"], case["op"]
    size = 4 if case["dtype"] == "float32" else 2
    whole = n * L * C
    live = whole / 2 if case.get("ragged") else whole
    if op in ("norm", "norm_back"):
        reads, writes, flops = (1, 1, 10) if op == "norm" else (2, 1, 24)
        small = (8 if op == "norm" else 16) * C + 8 * n * case["groups"]
    elif op in ("rec", "rec_step"):
        reads, writes, flops = (3, 1, 10) if case["gate"] else (2, 1, 7)
        small = 4 * ((2 if case["state"] else 1) + (-(-L // EVERY) if case["keep"] else 0)) * n * C
    elif op == "rec_back":
        reads, writes, flops = (4, 3, 26) if case["gate"] else (3, 2, 18)
        small = 4 * ((2 if case["state"] else 1) + -(-L // EVERY)) * n * C
    else:
        reads, writes, flops, small = (2 if case["residual"] else 1), 1, 15, 0
    return dict(bytes=int((reads * live + writes * whole) * size + small), flops=int(flops * live))


# --------------------------------------------------- the definitions, 64 bits
def _logistic(x):
    return torch.sigmoid(x.double())


def _exact_norm(s):
    case, x = s["case"], s["x"]
    n, L, C = x.shape
    G, act = case["groups"], case["act"]
    w, b = s["weight"].double(), s["bias"].double()
    y = torch.zeros((n, L, C), dtype=torch.float64, device=x.device)
    mean = torch.zeros((n, G), dtype=torch.float64, device=x.device)
    rstd = torch.zeros_like(mean)
    lens = [L] * n if s["lengths"] is None else s["lengths"].tolist()
    for i, T in enumerate(lens):
        if T == 0:
            continue
        xi = x[i, :T].double().view(T, G, C // G).transpose(0, 1).reshape(G, -1)
        mean[i] = xi.mean(1)
        rstd[i] = (xi.var(1, unbiased=False) + EPS).rsqrt()
        xh = ((xi - mean[i][:, None]) * rstd[i][:, None]).view(G, T, C // G).transpose(0, 1).reshape(T, C)
        z = xh * w + b
        if act == "relu":
            z = z.clamp(min=0.0)
        elif act == "silu":
            z = z * torch.sigmoid(z)
        elif act == "gelu":
            z = z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        y[i, :T] = z
    return dict(y=y, mean=mean, rstd=rstd)


def _exact_norm_back(s):
    case, x = s["case"], s["x"]
    n, L, C = x.shape
    G, act = case["groups"], case["act"]
    w, b = s["weight"].double(), s["bias"].double()
    dx = torch.zeros((n, L, C), dtype=torch.float64, device=x.device)
    dweight, dbias = torch.zeros_like(w), torch.zeros_like(w)
    lens = [L] * n if s["lengths"] is None else s["lengths"].tolist()
    for i, T in enumerate(lens):
        if T == 0:
            continue
        m = s["mean"][i].double().repeat_interleave(C // G)
        r = s["rstd"][i].double().repeat_interleave(C // G)
        xh = (x[i, :T].double() - m) * r
        z = xh * w + b
        if act == "relu":
            slope = torch.where(z > 0, 1.0, 0.0)
        elif act == "silu":
            q = torch.sigmoid(z)
            slope = q + z * q * (1 - q)
        elif act == "gelu":
            slope = 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * (-z * z / 2).exp() / math.sqrt(2 * math.pi)
        else:
            slope = torch.ones_like(z)
        dz = s["dy"][i, :T].double() * slope
        dbias += dz.sum(0)
        dweight += (dz * xh).sum(0)
        g = dz * w
        mg = g.view(T, G, -1).mean(dim=(0, 2)).repeat_interleave(C // G)
        mgx = (g * xh).view(T, G, -1).mean(dim=(0, 2)).repeat_interleave(C // G)
        dx[i, :T] = r * (g - mg - xh * mgx)
    return dict(dx=dx, dweight=dweight, dbias=dbias)


def _exact_states(s, L):
    """h before step 0 and after every step, [L + 1] of [n, C], step by step."""
    v, f = s["v"], s["f"]
    h = torch.zeros(v.shape[0], v.shape[2], dtype=torch.float64, device=v.device)
    if s["h0"] is not None:
        h = s["h0"].double()
    states = torch.empty((L + 1,) + tuple(h.shape), dtype=torch.float64, device=v.device)
    states[0] = h
    for t in range(L):
        a = _logistic(f[:, t])
        new = v[:, t] + a * (h - v[:, t])
        if s["lengths"] is not None:
            new = torch.where((s["lengths"] > t)[:, None], new, h)
        h = new
        states[t + 1] = h
    return states


def _exact_rec(s):
    n, L, C = s["v"].shape
    states = _exact_states(s, L)
    y = states[1:].transpose(0, 1)
    if s["o"] is not None:
        y = y * _logistic(s["o"])
    if s["lengths"] is not None:
        y = y.masked_fill((torch.arange(L, device=y.device)[None, :] >= s["lengths"][:, None])[:, :, None], 0.0)
    out = dict(y=y, h_last=states[L].clone())
    if s["case"]["keep"]:
        out["states"] = states[0:L:EVERY].transpose(0, 1).contiguous()
    return out


def _exact_rec_back(s):
    n, L, C = s["v"].shape
    states = _exact_states(s, L)
    shape, dev = (n, L, C), s["v"].device
    dv, df, do = (torch.zeros(shape, dtype=torch.float64, device=dev) for _ in range(3))
    dh = torch.zeros((n, C), dtype=torch.float64, device=dev) if s["dh_last"] is None else s["dh_last"].double()
    zero = torch.zeros((), dtype=torch.float64, device=dev)
    for t in range(L - 1, -1, -1):
        on = None if s["lengths"] is None else (s["lengths"] > t)[:, None]
        a, g = _logistic(s["f"][:, t]), s["dy"][:, t].double()
        if s["o"] is not None:
            q = _logistic(s["o"][:, t])
            d = g * states[t + 1] * q * (1 - q)
            do[:, t] = d if on is None else torch.where(on, d, zero)
            g = g * q
        total = dh + g
        dvt, dft = total * (1 - a), total * (states[t] - s["v"][:, t]) * a * (1 - a)
        if on is None:
            dv[:, t], df[:, t], dh = dvt, dft, total * a
        else:
            dv[:, t], df[:, t] = torch.where(on, dvt, zero), torch.where(on, dft, zero)
            dh = torch.where(on, total * a, dh)
    out = dict(dv=dv, df=df, dh0=dh)
    return out if s["o"] is None else dict(out, do=do)


def _exact_rec_step(s):
    a = _logistic(s["f"])
    h = s["v"] + a * (s["h"].double() - s["v"])
    return dict(y=h if s["o"] is None else h * _logistic(s["o"]), h=h)


def _exact_drop(s):
    """Philox with the 32-bit factors in 16-bit limbs, block by block of the flat tensor."""
    case, x = s["case"], s["x"]
    d = _threshold(case["p"])
    flat = x.reshape(-1)
    res = None if s["residual"] is None else s["residual"].reshape(-1)
    y = torch.zeros(flat.shape, dtype=torch.float64, device=x.device)

    def both_halves(u, const):
        ul, uh, cl, ch = u & 0xFFFF, u >> 16, const & 0xFFFF, const >> 16
        mid = (ul * cl >> 16) + (uh * cl & 0xFFFF) + (ul * ch & 0xFFFF)
        high = uh * ch + (uh * cl >> 16) + (ul * ch >> 16) + (mid >> 16)
        return high, (mid & 0xFFFF) << 16 | (ul * cl & 0xFFFF)

    step = 1 << 25
    for at in range(0, flat.numel(), step):
        end = min(flat.numel(), at + step)
        i = torch.arange(at // 8, (end + 7) // 8, device=x.device)
        w0, w1 = i % (1 << 32), i // (1 << 32)
        w2, w3 = torch.full_like(i, case["call"] % (1 << 32)), torch.full_like(i, case["call"] // (1 << 32))
        for r in range(10):
            key0 = (s["seed"] % (1 << 32) + r * 0x9E3779B9) % (1 << 32)
            key1 = (s["seed"] // (1 << 32) + r * 0xBB67AE85) % (1 << 32)
            h0, l0 = both_halves(w0, 0xD2511F53)
            h1, l1 = both_halves(w2, 0xCD9E8D57)
            w0, w1, w2, w3 = h1 ^ w1 ^ key0, l1, h0 ^ w3 ^ key1, l0
        u = torch.empty((i.numel(), 8), dtype=torch.int64, device=x.device)
        for k, w in enumerate((w0, w1, w2, w3)):
            u[:, 2 * k], u[:, 2 * k + 1] = w % 65536, w // 65536
        drop = u.view(-1)[:end - at] < d
        part = (flat[at:end].double() * (65536 / max(1, 65536 - d))).masked_fill(drop, 0.0)
        y[at:end] = part if res is None else part + res[at:end].double()
    return y.view(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    return dict(norm=_exact_norm, norm_back=_exact_norm_back, rec=_exact_rec, rec_back=_exact_rec_back,
                rec_step=_exact_rec_step, drop=_exact_drop, drop_back=_exact_drop)[case["op"]](s)
