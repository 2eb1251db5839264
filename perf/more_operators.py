"""The cases on which the root-mean-square norm, the causal convolution with the
selective state space scan, and beam search's selection with the reordering of
states are timed, with plain forms of each.

Sizes are those of the library's own workloads where there is one (widths 1024,
2048, 2560, 4096, 8192, the 32001 rows of an output layer, sequences of 65536
steps) and generic ones elsewhere.
"""
import math

import torch

own = False  # True: run() calls the library; False: the plain form

EPS = 1e-5


# ---------------------------------------------------------------- cases
def listed():
    return [
        # Serving: one token for each of 32 sequences; the last product's fp32 output joins a bf16 residual.
        dict(name="norm_one_token_32", op="norm", T=32, D=4096, x="fp32", r="bf16", res=True, y="bf16"),
        # A long prompt whose next product is block-scaled: the norm writes E4M3 and the scales.
        dict(name="norm_prompt_mx", op="norm", T=8192, D=4096, x="fp32", r="bf16", res=True, y="mx"),
        # A training step's backward pass, the residual's gradient joining.
        dict(name="norm_bwd_train", op="normb", T=16384, D=2560, r="bf16", g="bf16", dres=True),
        # Serving: the convolution of one token for 64 sequences, x half of a projection's rows.
        dict(name="conv_one_token_64", op="convs", batch=64, C=5120, width=4, slots=80, x="fp32", y="bf16", wide=True),
        # A batch of prompts.
        dict(name="conv_prompt", op="conv", T=2048, batch=8, C=4096, width=4, x="bf16", y="bf16", wide=True, ragged=False),
        # Serving: one token for 64 sequences whose states sit in a cache of 80 slots.
        dict(name="scan_one_token_64", op="scans", batch=64, C=5120, N=16, slots=80, u="bf16", p="fp32", gate=True),
        # A batch of prompts, the operands as the projections leave them.
        dict(name="scan_prompt", op="scan", T=2048, batch=8, C=4096, N=16, u="bf16", p="fp32", gate=True, ragged=False),
        # One long document: few channels, so the work has to be split over time.
        dict(name="scan_long", op="scan", T=65536, batch=1, C=1024, N=16, u="bf16", p="bf16", gate=True, ragged=False),
        # A padded batch of odd width: sequences of length 0 and 1 among longer ones.
        dict(name="scan_ragged_odd", op="scan", T=777, batch=6, C=1001, N=12, u="fp32", p="fp32", gate=False, ragged=True),
        # One request searched with four beams over an output layer of odd height.
        dict(name="beam_select_one", op="select", batch=1, beams=4, V=32001, count=4, logits="fp32", ends=False),
        # Many requests, wide vocabulary; twice as many candidates as beams, for sequences that end.
        dict(name="beam_select_many", op="select", batch=64, beams=8, V=128000, count=16, logits="fp32", ends=True),
        # Their states follow the chosen beams: 24 layers of scan states.
        dict(name="beam_reorder", op="reorder", layers=24, batch=8, beams=8, row=32768, slots=70, kind="fp32"),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    v = min(max(v, -(-lo // step) * step), hi // step * step)
    return v


def draw(rng):
    op = rng.choice(("norm", "norm", "normb", "convs", "conv", "scans", "scan", "scan", "select", "select", "reorder"))
    kinds = ("bf16", "fp32")
    if op in ("norm", "normb"):
        D = _log(rng, 64, 16384, rng.choice((1, 8, 32)))
        T = _log(rng, 1, min(16384, 33_500_000 // D))
        if op == "norm":
            return dict(op=op, T=T, D=D, x=rng.choice(kinds), r=rng.choice(kinds), res=rng.random() < 0.8,
                        y=rng.choice(("bf16", "mx", "fp32")))
        return dict(op=op, T=T, D=D, r=rng.choice(kinds), g=rng.choice(kinds), dres=rng.random() < 0.7)
    if op == "convs":
        batch = _log(rng, 1, 256)
        return dict(op=op, batch=batch, C=_log(rng, 64, 10240, rng.choice((1, 8))), width=rng.randint(2, 4),
                    slots=batch + rng.randrange(64), x=rng.choice(kinds), y=rng.choice(kinds), wide=rng.random() < 0.5)
    if op == "conv":
        C = _log(rng, 64, 8192, rng.choice((1, 8)))
        batch = _log(rng, 1, 64)
        T = _log(rng, 1, max(1, min(65536, 33_000_000 // (C * batch))))
        return dict(op=op, T=T, batch=batch, C=C, width=rng.randint(2, 4), x=rng.choice(kinds), y=rng.choice(kinds),
                    wide=rng.random() < 0.5, ragged=rng.random() < 0.5)
    if op == "scans":
        batch = _log(rng, 1, 256)
        return dict(op=op, batch=batch, C=_log(rng, 64, 5120), N=rng.choice((1, 8, 12, 16, 16, 16)),
                    slots=batch + rng.randrange(64), u=rng.choice(kinds), p=rng.choice(kinds), gate=rng.random() < 0.7)
    if op == "scan":
        C = _log(rng, 64, 5120)
        N = rng.choice((1, 8, 12, 16, 16, 16, 32, 64, 128))
        batch = _log(rng, 1, max(1, min(64, 500_000_000 // (C * N))))
        T = _log(rng, 1, max(1, min(65536, 60_000_000 // (C * batch), 1_000_000_000 // (C * N * batch))))
        return dict(op=op, T=T, batch=batch, C=C, N=N, u=rng.choice(kinds), p=rng.choice(kinds),
                    gate=rng.random() < 0.7, ragged=rng.random() < 0.5)
    if op == "select":
        beams = rng.randint(1, 16)
        V = _log(rng, 512, 128000)
        batch = _log(rng, 1, max(1, min(64, 65_000_000 // (beams * V))))
        return dict(op=op, batch=batch, beams=beams, V=V, count=beams * rng.choice((1, 2)), logits=rng.choice(kinds),
                    ends=rng.random() < 0.5)
    layers, batch, beams = _log(rng, 1, 48), _log(rng, 1, 64), rng.randint(2, 16)
    row = _log(rng, 64, max(65, min(131072, 48_000_000 // (layers * batch * beams))))
    return dict(op=op, layers=layers, batch=batch, beams=beams, row=row, slots=batch * beams + rng.randrange(8),
                kind=rng.choice(kinds))


# ---------------------------------------------------------------- inputs
def _type(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _lengths(case):
    """A padded batch's lengths: the longest full, the others spread down to
    nothing, one of them empty and one of a single step where there are enough."""
    T, batch = case["T"], case["batch"]
    n = [T - (T * b) // batch for b in range(batch)]
    if batch > 2:
        n[1] = 0
    if batch > 3:
        n[2] = 1
    return n


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=gen, device="cuda").mul_(hi - lo).add_(lo)

    def ids(count, slots):
        i = torch.randperm(slots, generator=gen, device="cuda")[:count].to(torch.int32)
        if count > 3:
            i[count // 2] = -1  # a padding row of the batch
        return i

    op = case["op"]
    s = dict(case=case)
    if op == "norm":
        T, D = case["T"], case["D"]
        # A block's output and the residual stream: rows of differing size, a few channels far larger than the rest.
        big = 1.0 + 20.0 * (uniform(0, 1, D) < 0.01)
        s["x"] = (normal(T, D) * big).to(_type(case["x"]))
        s["res"] = (normal(T, D) * big * uniform(0.5, 4.0, T, 1)).to(_type(case["r"])) if case["res"] else None
        s["res_out"] = torch.empty(T, D, dtype=_type(case["r"]), device="cuda") if case["res"] else None
        s["w"] = uniform(0.2, 1.8, D)
        mx = case["y"] == "mx"
        s["y"] = None if mx else torch.empty(T, D, dtype=_type(case["y"]), device="cuda")
        s["y8"] = torch.empty(T, D, dtype=torch.uint8, device="cuda") if mx else None
        s["y8_scales"] = torch.empty(-(-D // 128), T, 4, dtype=torch.uint8, device="cuda") if mx else None
    elif op == "normb":
        T, D = case["T"], case["D"]
        big = 1.0 + 20.0 * (uniform(0, 1, D) < 0.01)
        s["r"] = (normal(T, D) * big * uniform(0.5, 4.0, T, 1)).to(_type(case["r"]))
        s["w"] = uniform(0.2, 1.8, D)
        s["dy"] = normal(T, D).to(_type(case["g"]))
        s["dres"] = normal(T, D).to(_type(case["g"])) if case["dres"] else None
        s["dx"] = torch.empty(T, D, dtype=_type(case["g"]), device="cuda")
        s["dw"] = torch.empty(D, device="cuda")
    elif op in ("conv", "convs"):
        C, width = case["C"], case["width"]
        rows = (case["T"], case["batch"]) if op == "conv" else (case["batch"],)
        xz = normal(*rows, 2 * C if case["wide"] else C).to(_type(case["x"]))
        s["x"] = xz[..., :C]  # a view of a projection's rows, which hold the gate too
        s["w"] = uniform(-1, 1, width, C) / math.sqrt(width)
        s["bias"] = uniform(-0.5, 0.5, C)
        s["y"] = torch.empty(*rows, C, dtype=_type(case["y"]), device="cuda")
        if op == "conv":
            s["lengths"] = None
            if case["ragged"]:
                s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
                live = torch.arange(case["T"], device="cuda")[:, None, None] < s["lengths"][None, :, None]
                xz.masked_fill_(~live, float("nan"))  # padding holds anything
            s["state"] = normal(case["batch"], width - 1, C).to(_type(case["x"]))
            s["new_state"] = torch.empty_like(s["state"])
        else:
            s["slot_ids"] = ids(case["batch"], case["slots"])
            s["state"] = normal(case["slots"], width - 1, C).to(_type(case["x"]))
            s["new_state"] = s["state"].clone()
    elif op in ("scan", "scans"):
        C, N = case["C"], case["N"]
        rows = (case["T"], case["batch"]) if op == "scan" else (case["batch"],)
        p = _type(case["p"])
        s["u"] = (normal(*rows, C) * torch.rand(C, generator=gen, device="cuda")).to(_type(case["u"]))
        # dt's bias is set so that softplus(bias) spreads over 0.001 to 0.1; A[c][n] = -(n + 1), learned on from there.
        step = torch.exp(uniform(math.log(1e-3), math.log(0.1), C))
        s["dt_bias"] = step + torch.log(-torch.expm1(-step))
        s["dt"] = normal(*rows, C).to(p)
        s["A"] = -torch.arange(1, N + 1, device="cuda") * uniform(0.8, 1.25, C, N)
        s["D"] = normal(C)
        s["bc"] = normal(*rows, 2 * N).to(p)  # B and C: columns of one projection's rows
        xz = normal(*rows, 2 * C).to(p) if case["gate"] else None
        s["z"] = xz[..., C:] if case["gate"] else None  # the gate: the other half of the first projection's rows
        s["y"] = torch.empty(*rows, C, dtype=_type(case["u"]), device="cuda")
        if op == "scan":
            s["lengths"] = None
            if case["ragged"]:
                s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
                live = torch.arange(case["T"], device="cuda")[:, None, None] < s["lengths"][None, :, None]
                for name in ("u", "dt", "bc", "z"):
                    if s[name] is not None:
                        s[name].masked_fill_(~live, float("nan"))
            s["h0"] = normal(case["batch"], C, N)
            s["h_last"] = torch.empty_like(s["h0"])
        else:
            s["slot_ids"] = ids(case["batch"], case["slots"])
            s["state"] = normal(case["slots"], C, N)
            s["new_state"] = s["state"].clone()
    elif op == "select":
        batch, beams, V = case["batch"], case["beams"], case["V"]
        logits = normal(batch, beams, V).mul_(2.5)
        # Tokens that a grammar forbids.
        logits.masked_fill_(uniform(0, 1, batch, 1, V) < 0.05, -math.inf)
        s["logits"] = logits.to(_type(case["logits"]))
        s["scores"] = -torch.cumsum(uniform(0.0, 0.7, batch, beams), 1) - 3.0
        s["finished"], s["eos"] = None, -1
        if case["ends"]:
            s["finished"] = uniform(0, 1, batch, beams) < 0.15
            s["eos"] = 2
        n = case["count"]
        s["new_scores"] = torch.empty(batch, n, device="cuda")
        s["parents"] = torch.empty(batch, n, dtype=torch.int32, device="cuda")
        s["tokens"] = torch.empty(batch, n, dtype=torch.int32, device="cuda")
        s["new_finished"] = torch.empty(batch, n, dtype=torch.bool, device="cuda") if case["ends"] else None
    else:
        layers, batch, beams = case["layers"], case["batch"], case["beams"]
        s["state"] = normal(layers, case["slots"], case["row"]).to(_type(case["kind"]))
        s["slot_ids"] = torch.randperm(case["slots"], generator=gen, device="cuda")[: batch * beams].to(torch.int32)
        s["parents"] = torch.randint(0, beams, (batch, beams), generator=gen, device="cuda", dtype=torch.int32)
        s["new_state"] = s["state"].clone()
    return s


# ---------------------------------------------------------------- plain forms (32 bits)
def _norm(x, res, w, r_type):
    r = x.float() + (0.0 if res is None else res.float())
    y = r * torch.rsqrt((r * r).mean(dim=1, keepdim=True) + EPS) * w
    return y, (None if res is None else r.to(r_type))


def _mx(y):
    """E4M3 values and E8M0 scales of blocks of 32: the least power of two that leaves no value above 448."""
    T, D = y.shape
    atoms = -(-D // 128)
    v = torch.zeros(T, atoms * 128, dtype=y.dtype, device=y.device)
    v[:, :D] = y
    v = v.view(T, atoms * 4, 32)
    m, e = torch.frexp(v.abs().amax(dim=2))
    e = torch.where(m > 0, e - 9 + (m > 0.875), -127).clamp(-127, 127)
    q = torch.ldexp(v, -e[:, :, None]).to(torch.float8_e4m3fn).view(T, -1)[:, :D]
    scales = (e + 127).to(torch.uint8).view(T, atoms, 4).transpose(0, 1)
    return q.contiguous(), scales.contiguous().view(torch.float8_e8m0fnu)


def _norm_backward(r, w, dy, dres):
    r, dy = r.float(), dy.float()
    k = torch.rsqrt((r * r).mean(dim=1, keepdim=True) + EPS)
    n, d = r * k, dy * w
    dx = k * (d - n * (d * n).mean(dim=1, keepdim=True))
    if dres is not None:
        dx = dx + dres.float()
    return dx, (dy * n).sum(dim=0)


def _silu(v):
    return v * torch.sigmoid(v)


def _conv(x, w, bias, state, lengths):
    """x [T,batch,C], state [batch,width-1,C]; outputs and the inputs that the next step needs."""
    T, batch, C = x.shape
    width = w.shape[0]
    before = torch.cat([state.transpose(0, 1), x])  # step t's taps are rows t .. t + width - 1
    taps = torch.stack([before[j: j + T].float() * w[j] for j in range(width)])
    y = _silu(taps.sum(dim=0) + bias)
    if lengths is None:
        return y, before[T:].transpose(0, 1).contiguous()
    live = torch.arange(T, device=x.device)[:, None, None] < lengths[None, :, None]
    at = lengths.long()[:, None] + torch.arange(width - 1, device=x.device)
    last = before[at, torch.arange(batch, device=x.device)[:, None]]
    return torch.where(live, y, 0.0), last


def _conv_step(x, w, bias, slot_ids, state):
    used = slot_ids >= 0
    at = slot_ids.clamp(min=0).long()
    window = torch.cat([state[at], x[:, None]], dim=1)
    y = _silu((window.float() * w).sum(dim=1) + bias)
    new = torch.cat([state, state[:1]])  # a last row takes what padding rows write
    new[torch.where(used, at, state.shape[0])] = window[:, 1:]
    return torch.where(used[:, None], y, 0.0), new[:-1]


def _scan(a, b):
    """All prefixes of h -> a h + b along the first axis, doubling the distance."""
    d = 1
    while d < a.shape[0]:
        b = torch.cat([b[:d], a[d:] * b[:-d] + b[d:]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _softplus(v):
    return torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-v.abs()))


def _selective(u, dt, dt_bias, A, bc, D, z, h0, lengths):
    """u, dt [T,batch,C], A [C,N], bc [T,batch,2N], h0 [batch,C,N]."""
    N = A.shape[1]
    u, delta, B, Cm = u.float(), _softplus(dt.float() + dt_bias), bc[..., :N].float(), bc[..., N:].float()
    live = None
    if lengths is not None:
        live = torch.arange(u.shape[0], device=u.device)[:, None, None] < lengths[None, :, None]
        u, delta, B, Cm = (torch.where(live, v, 0.0) for v in (u, delta, B, Cm))
    a = torch.exp(delta[..., None] * A)
    b = (delta * u)[..., None] * B[:, :, None, :]
    b[0] += a[0] * h0
    h = _scan(a, b)
    y = (h * Cm[:, :, None, :]).sum(dim=3) + D * u
    if z is not None:
        y = y * _silu(z.float())
    if live is not None:
        y = torch.where(live, y, 0.0)
    return y, h[-1].clone()


def _selective_step(u, dt, dt_bias, A, bc, D, z, slot_ids, state):
    N = A.shape[1]
    used = slot_ids >= 0
    at = slot_ids.clamp(min=0).long()
    u, delta, B, Cm = u.float(), _softplus(dt.float() + dt_bias), bc[..., :N].float(), bc[..., N:].float()
    h = torch.exp(delta[..., None] * A) * state[at] + (delta * u)[..., None] * B[:, None, :]
    y = (h * Cm[:, None, :]).sum(dim=2) + D * u
    if z is not None:
        y = y * _silu(z.float())
    new = torch.cat([state, state[:1]])
    new[torch.where(used, at, state.shape[0])] = h
    return torch.where(used[:, None], y, 0.0), new[:-1]


def _select(logits, scores, finished, eos, count):
    """The `count` best continuations of each sequence's beams, best first; a row's
    own order is by logit and then token, a sequence's by score and then beam."""
    batch, beams, V = logits.shape
    l = logits.float() + 0.0
    # Whole numbers in the order of (logit, lower token first).
    bits = l.view(torch.int32)
    key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32) | (0x7FFFFFFF - torch.arange(V, device=l.device))
    n = min(count, V)
    token = 0x7FFFFFFF - (torch.topk(key, n, dim=2).values & 0xFFFFFFFF)
    best = torch.gather(l, 2, token).double()
    top = best[..., :1]
    score = scores.double()[..., None] + (best - top - torch.log(torch.exp(l.double() - top).sum(dim=2, keepdim=True)))
    if finished is not None:
        first = torch.arange(n, device=l.device) == 0
        ended = torch.where(first, scores.double()[..., None], -math.inf)
        score = torch.where(finished[..., None], ended, score)
        token = torch.where(finished[..., None], eos, token)
    score, at = torch.sort(score.view(batch, -1), dim=1, descending=True, stable=True)
    score, at = score[:, :count], at[:, :count]
    parent, token = at // n, torch.gather(token.view(batch, -1), 1, at)
    found = score > -math.inf  # places that no candidate fills: beam 0, token 0
    parent, token = torch.where(found, parent, 0), torch.where(found, token, 0)
    out = score.float(), parent.to(torch.int32), token.to(torch.int32)
    if finished is None:
        return out
    return *out, found & (torch.gather(finished, 1, parent) | (token == eos))


def _reorder(state, slot_ids, parents):
    batch, beams = parents.shape
    ids = slot_ids.long().view(batch, beams)
    new = state.clone()
    new[:, ids.view(-1)] = state[:, torch.gather(ids, 1, parents.long()).view(-1)]
    return new


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_1810_09958_gb300 import isam
        if op == "norm":
            isam.rms_norm_forward(case["T"], case["D"], s["x"], s["res"], s["res_out"], s["w"], EPS, s["y"], s["y8"],
                                  s["y8_scales"])
            if s["y"] is None:
                return s["y8"].view(torch.float8_e4m3fn), s["y8_scales"].view(torch.float8_e8m0fnu), s["res_out"]
            return s["y"], s["res_out"]
        if op == "normb":
            isam.rms_norm_backward(case["T"], case["D"], s["r"], s["w"], EPS, s["dy"], s["dres"], s["dx"], s["dw"])
            return s["dx"], s["dw"]
        if op == "conv":
            isam.conv1d_forward(case["T"], case["batch"], case["C"], case["width"], s["x"], s["w"], s["bias"], True,
                                s["state"], s["lengths"], s["y"], s["new_state"])
            return s["y"], s["new_state"]
        if op == "convs":
            isam.conv1d_step(case["batch"], case["C"], case["width"], case["slots"], s["x"], s["w"], s["bias"], True,
                             s["slot_ids"], s["state"], s["new_state"], s["y"])
            return s["y"], s["new_state"]
        if op in ("scan", "scans"):
            N = case["N"]
            B, Cm = s["bc"][..., :N], s["bc"][..., N:]
            if op == "scan":
                isam.ssm_forward(case["T"], case["batch"], case["C"], N, s["u"], s["dt"], s["dt_bias"], s["A"], B, Cm,
                                 s["D"], s["z"], s["h0"], s["lengths"], s["y"], s["h_last"])
                return s["y"], s["h_last"]
            isam.ssm_step(case["batch"], case["C"], N, case["slots"], s["u"], s["dt"], s["dt_bias"], s["A"], B, Cm,
                          s["D"], s["z"], s["slot_ids"], s["state"], s["new_state"], s["y"])
            return s["y"], s["new_state"]
        if op == "select":
            isam.beam_select(case["batch"], case["beams"], case["V"], case["count"], s["logits"], s["scores"], s["eos"],
                             s["finished"], s["new_scores"], s["parents"], s["tokens"], s["new_finished"])
            out = s["new_scores"], s["parents"], s["tokens"]
            return out if s["finished"] is None else (*out, s["new_finished"])
        isam.beam_reorder(case["layers"], case["batch"], case["beams"], case["slots"], s["parents"], s["slot_ids"],
                          s["state"], s["new_state"])
        return s["new_state"]
    if op == "norm":
        y, r = _norm(s["x"], s["res"], s["w"], _type(case["r"]))
        return (*_mx(y), r) if case["y"] == "mx" else (y.to(_type(case["y"])), r)
    if op == "normb":
        dx, dw = _norm_backward(s["r"], s["w"], s["dy"], s["dres"])
        return dx.to(_type(case["g"])), dw
    if op == "conv":
        y, last = _conv(s["x"], s["w"], s["bias"], s["state"], s["lengths"])
        return y.to(_type(case["y"])), last
    if op == "convs":
        y, new = _conv_step(s["x"], s["w"], s["bias"], s["slot_ids"], s["state"])
        return y.to(_type(case["y"])), new
    if op == "scan":
        y, last = _selective(s["u"], s["dt"], s["dt_bias"], s["A"], s["bc"], s["D"], s["z"], s["h0"], s["lengths"])
        return y.to(_type(case["u"])), last
    if op == "scans":
        y, new = _selective_step(s["u"], s["dt"], s["dt_bias"], s["A"], s["bc"], s["D"], s["z"], s["slot_ids"],
                                 s["state"])
        return y.to(_type(case["u"])), new
    if op == "select":
        return _select(s["logits"], s["scores"], s["finished"], s["eos"], case["count"])
    return _reorder(s["state"], s["slot_ids"], s["parents"])


def work(case):
    op = case["op"]
    size = {"bf16": 2, "fp32": 4}
    if op == "norm":
        n = case["T"] * case["D"]
        y = 1 + 1 / 32 if case["y"] == "mx" else size[case["y"]]
        return dict(bytes=n * (size[case["x"]] + (2 * size[case["r"]] if case["res"] else 0) + y) + 4.0 * case["D"],
                    flops=6.0 * n)
    if op == "normb":
        n = case["T"] * case["D"]
        return dict(bytes=n * (size[case["r"]] + size[case["g"]] * (3 if case["dres"] else 2)) + 8.0 * case["D"],
                    flops=12.0 * n)
    if op in ("conv", "convs"):
        # A padded batch reads its live steps alone, and writes the zeros of the others too.
        C, width, batch = case["C"], case["width"], case["batch"]
        n = case.get("T", 1) * batch * C
        live = sum(_lengths(case)) * C if case.get("ragged") else n
        x = size[case["x"]]
        return dict(bytes=live * x + n * size[case["y"]] + 2.0 * batch * (width - 1) * C * x + 4.0 * (width + 1) * C,
                    flops=(2.0 * width + 6) * live)
    if op in ("scan", "scans"):
        C, N, batch = case["C"], case["N"], case["batch"]
        n = case.get("T", 1) * batch * C
        live = sum(_lengths(case)) * C if case.get("ragged") else n
        u, p = size[case["u"]], size[case["p"]]
        return dict(bytes=live * (u + (2 if case["gate"] else 1) * p) + n * u + live // C * 2.0 * N * p
                    + 8.0 * batch * C * N + 4.0 * C * (N + 2), flops=live * (7.0 * N + 16))
    if op == "select":
        rows, n = case["batch"] * case["beams"], case["batch"] * case["count"]
        return dict(bytes=float(rows) * case["V"] * size[case["logits"]] + 4.0 * rows + 12.0 * n,
                    flops=3.0 * rows * case["V"])
    n = case["layers"] * case["batch"] * case["beams"] * case["row"]
    return dict(bytes=2.0 * n * size[case["kind"]], flops=0.0)


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The definitions, step by step, in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        r = s["x"].double()
        if s["res"] is not None:
            r = r + s["res"].double()
        y = r / torch.sqrt(r.square().sum(dim=1, keepdim=True) / case["D"] + EPS) * s["w"].double()
        r = r if s["res"] is not None else None
        if case["y"] != "mx":
            return y, r
        # Each value over its block's scale, before it is rounded to 8 bits; a scale is a border's choice.
        for at in range(0, case["D"], 32):
            block = y[:, at: at + 32]
            top = block.abs().amax(dim=1, keepdim=True)
            block /= torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).clamp(-127, 127))
        return y, None, r
    if op == "normb":
        r, w, dy = s["r"].double(), s["w"].double(), s["dy"].double()
        k = 1 / torch.sqrt(r.square().sum(dim=1, keepdim=True) / case["D"] + EPS)
        # y_j = w_j r_j k: dy_j / dr_i = w_j (k [i = j] - r_j k^3 r_i / D)
        dx = k * w * dy - k ** 3 * r / case["D"] * (w * dy * r).sum(dim=1, keepdim=True)
        if s["dres"] is not None:
            dx += s["dres"].double()
        return dx, (dy * r * k).sum(dim=0)
    if op in ("conv", "convs"):
        width, w, bias = case["width"], s["w"].double(), s["bias"].double()
        if op == "convs":
            y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
            new = s["state"].double()
            for i, slot in enumerate(s["slot_ids"].tolist()):
                if slot >= 0:
                    window = torch.cat([new[slot], s["x"][i: i + 1].double()])
                    v = bias + sum(window[j] * w[j] for j in range(width))
                    y[i] = v / (1 + torch.exp(-v))
                    new[slot] = window[1:]
            return y, new
        T = case["T"]
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        new = s["state"].double()
        for b, n in enumerate([T] * case["batch"] if s["lengths"] is None else s["lengths"].tolist()):
            line = torch.cat([new[b], s["x"][:n, b].double()])
            v = bias.expand(n, -1).clone()
            for j in range(width):
                v += line[j: j + n] * w[j]
            y[:n, b] = v / (1 + torch.exp(-v))
            new[b] = line[n:]
        return y, new
    if op in ("scan", "scans"):
        N, A, D, bias = case["N"], s["A"].double(), s["D"].double(), s["dt_bias"].double()

        def rows(at):
            """u, delta, B, C and the gate of some rows."""
            v = s["dt"][at].double() + bias
            bc = s["bc"][at].double()
            delta = torch.where(v > 30, v, torch.log1p(torch.exp(v.clamp(max=30))))
            z = torch.ones_like(v)
            if s["z"] is not None:
                z = s["z"][at].double()
                z = z / (1 + torch.exp(-z))
            return s["u"][at].double(), delta, bc[..., None, :N], bc[..., None, N:], z

        if op == "scans":
            at = s["slot_ids"].long()
            used = at >= 0
            u, delta, B, Cm, z = rows(slice(None))
            h = torch.exp(delta[..., None] * A) * s["state"].double()[at.clamp(min=0)] + (delta * u)[..., None] * B
            y = ((h * Cm).sum(dim=2) + D * u) * z
            new = s["state"].double()
            new[at[used]] = h[used]
            y[~used] = 0.0
            return y, new
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        h = s["h0"].double()
        for first in range(0, case["T"], 64):
            u, delta, B, Cm, z = rows(slice(first, first + 64))
            for i in range(u.shape[0]):
                new = torch.exp(delta[i, ..., None] * A).mul_(h).addcmul_((delta[i] * u[i])[..., None], B[i])
                out = (new * Cm[i]).sum(dim=2)
                if s["lengths"] is None:
                    h, y[first + i] = new, out
                else:
                    on = (s["lengths"] > first + i)[:, None]
                    h, y[first + i] = torch.where(on[..., None], new, h), torch.where(on, out, 0.0)
            y[first: first + 64] = (y[first: first + 64] + D * u) * z
        if s["lengths"] is not None:
            y.masked_fill_(torch.arange(case["T"], device="cuda")[:, None, None] >= s["lengths"][:, None], 0.0)
        return y, h
    if op == "select":
        batch, beams, V, count = case["batch"], case["beams"], case["V"], case["count"]
        out = torch.empty(batch, count, dtype=torch.float64, device="cuda")
        for b in range(batch):
            l = s["logits"][b].double()
            p = s["scores"][b].double()[:, None] + l - torch.logsumexp(l, dim=1, keepdim=True)
            if s["finished"] is not None:
                ended = s["finished"][b]
                p[ended] = -math.inf
                p[ended, s["eos"]] = s["scores"][b].double()[ended]
            best = torch.sort(p.view(-1), descending=True).values[:count]
            out[b] = best
        return (out, None, None) if s["finished"] is None else (out, None, None, None)
    ids, new = s["slot_ids"].view(case["batch"], case["beams"]).tolist(), s["state"].double()
    parents = s["parents"].tolist()
    old = s["state"].double()
    for b, row in enumerate(ids):
        for k, slot in enumerate(row):
            new[:, slot] = old[:, row[parents[b][k]]]
    return new
