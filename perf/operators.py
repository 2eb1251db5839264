"""The cases on which the gated linear recurrence, the gated feed-forward
product and the 4-bit few-token product are timed, with plain forms of each.

Sizes are those of the library's own workloads where there is one (hidden
1024 and 128 steps of 32 sequences, the (M, K) pairs of the skinny GEMM sweep,
8192) and generic ones elsewhere.
"""
import math

import torch

own = False  # True: run() calls the library; False: the plain form

ACTS = ("silu", "gelu", "relu", "sigmoid")
NIBBLES = (0, 2, 4, 6, 1, 3, 5, 7)  # k offset held by each nibble of a 32-bit code word


# ---------------------------------------------------------------- cases
def listed():
    return [
        # Serving: one token for each of 32 sequences whose states sit in a cache of 64 slots.
        dict(name="recurrence_step_32", op="step", batch=32, hidden=1024, slots=64, g="bf16", h="bf16"),
        # The GRU benchmark's shape, fed by a projection's fp32 output and read by the next product.
        dict(name="recurrence_fwd_128x32x1024", op="rfwd", T=128, batch=32, hidden=1024, g="fp32", h="bf16", ragged=False),
        # A padded batch of odd width: sequences of length 0 and 1 among longer ones.
        dict(name="recurrence_fwd_ragged_odd", op="rfwd", T=777, batch=6, hidden=1001, g="fp32", h="fp32", ragged=True),
        # One long document: few channels, so the work has to be split over time.
        dict(name="recurrence_fwd_long", op="rfwd", T=65536, batch=1, hidden=2560, g="bf16", h="bf16", ragged=False),
        # A training batch.
        dict(name="recurrence_bwd_train", op="rbwd", T=4096, batch=8, hidden=1024, g="bf16", h="bf16", ragged=False),
        # Two long documents of different lengths in a padded batch.
        dict(name="recurrence_bwd_long_ragged", op="rbwd", T=20001, batch=2, hidden=1760, g="fp32", h="bf16", ragged=True),
        # Serving one sequence: both projections of a feed-forward block read once.
        dict(name="glu_fwd_one_token", op="gfwd", T=1, D=2560, F=7680, act="silu"),
        # A short prompt.
        dict(name="glu_fwd_prompt_200", op="gfwd", T=200, D=1760, F=4096, act="gelu"),
        # A training batch or long prompt: bound by the tensor cores.
        dict(name="glu_fwd_8192", op="gfwd", T=8192, D=4096, F=8192, act="silu"),
        # Its training step's backward pass.
        dict(name="glu_bwd_4096", op="gbwd", T=4096, D=2560, F=7680, act="silu"),
        # Serving with 4-bit weights: a square projection for one token ...
        dict(name="w4_one_token_4096", op="w4", M=1, N=4096, K=4096, group=128),
        # ... and an output layer of odd height for eight.
        dict(name="w4_eight_tokens_head", op="w4", M=8, N=32001, K=8192, group=32),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    v = min(max(v, -(-lo // step) * step), hi // step * step)
    return v - step if v == 3072 else v


def draw(rng):
    op = rng.choice(("step", "rfwd", "rfwd", "rbwd", "rbwd", "gfwd", "gfwd", "gbwd", "w4", "w4"))
    kinds = ("bf16", "fp32")
    if op == "step":
        batch = _log(rng, 1, 256)
        return dict(op=op, batch=batch, hidden=_log(rng, 64, 8192), slots=batch + rng.randrange(64),
                    g=rng.choice(kinds), h=rng.choice(kinds))
    if op in ("rfwd", "rbwd"):
        most = 120_000_000 if op == "rfwd" else 60_000_000
        hidden = _log(rng, 64, 4096)
        batch = _log(rng, 1, 64)
        T = _log(rng, 1, min(65536, most // (hidden * batch)))
        return dict(op=op, T=T, batch=batch, hidden=hidden, g=rng.choice(kinds), h=rng.choice(kinds),
                    ragged=rng.random() < 0.5)
    if op in ("gfwd", "gbwd"):
        D = _log(rng, 256, 4096, 8)
        F = _log(rng, 512, 8192, 8)
        T = _log(rng, 1, min(8192, int((6e11 if op == "gfwd" else 1.8e11) / (2.0 * D * F))))
        return dict(op=op, T=T, D=D, F=F, act=rng.choice(ACTS))
    return dict(op=op, M=_log(rng, 1, 32), N=_log(rng, 512, 32000), K=_log(rng, 256, 8192, 8),
                group=rng.choice((32, 64, 128)))


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

    op = case["op"]
    s = dict(case=case)
    if op == "step":
        B, H = case["batch"], case["hidden"]
        g = normal(B, 2 * H)
        g[:, :H] += 2.0
        s["g"] = g.to(_type(case["g"]))
        s["slot_ids"] = torch.randperm(case["slots"], generator=gen, device="cuda")[:B].to(torch.int32)
        if B > 3:
            s["slot_ids"][B // 2] = -1  # a padding row of the batch
        s["state"] = normal(case["slots"], H)
        s["new_state"] = s["state"].clone()
        s["h"] = torch.empty(B, H, dtype=_type(case["h"]), device="cuda")
    elif op in ("rfwd", "rbwd"):
        T, B, H = case["T"], case["batch"], case["hidden"]
        g = normal(T, B, 2 * H)
        # Update gates of trained models keep most of the state: sigmoid(2 + N(0, 1.5)).
        g[:, :, :H].mul_(1.5).add_(2.0)
        s["lengths"] = None
        live = None
        if case["ragged"]:
            s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
            live = torch.arange(T, device="cuda")[:, None, None] < s["lengths"][None, :, None]
            g.masked_fill_(~live, float("nan"))  # padding holds anything
        s["g"] = g.to(_type(case["g"]))
        del g
        s["h0"] = normal(B, H)
        s["h_out"] = torch.empty(T, B, H, dtype=_type(case["h"]), device="cuda")
        if op == "rfwd":
            s["h_last"] = torch.empty(B, H, device="cuda")
        else:
            s["h_out"].copy_(_recurrence(s["g"], s["h0"], s["lengths"], s["h_out"].dtype)[0])
            dh = normal(T, B, H)
            if live is not None:
                dh.masked_fill_(~live, float("nan"))
            s["dh_out"] = dh.to(_type(case["h"]))
            s["dh_last"] = normal(B, H)
            s["dg"] = torch.empty_like(s["g"])
            s["dh0"] = torch.empty(B, H, device="cuda")
    elif op in ("gfwd", "gbwd"):
        T, D, F = case["T"], case["D"], case["F"]
        s["x"] = normal(T, D).bfloat16()
        s["W"] = (normal(2 * F, D) / math.sqrt(D)).bfloat16()
        if op == "gfwd":
            s["h"] = torch.empty(T, F, dtype=torch.bfloat16, device="cuda")
        else:
            s["dh"] = normal(T, F).bfloat16()
            s["dx"] = torch.empty_like(s["x"])
            s["dW"] = torch.empty_like(s["W"])
    else:
        M, N, K, group = case["M"], case["N"], case["K"], case["group"]
        s["x"] = normal(M, K).bfloat16()
        # Codes of a weight matrix quantised with its group's largest value at 8: N(0, 2.7), rounded and clipped.
        q = normal(N, K).mul_(2.7).round_().add_(8).clamp_(0, 15).to(torch.uint8)
        groups = -(-K // group)
        sc = (torch.rand(N, groups, generator=gen, device="cuda").mul_(0.01).add_(0.002)).bfloat16()
        s["codes"] = q[:, 0::2] | (q[:, 1::2] << 4)  # [N][K/2], the even k in the low half
        s["scales"] = sc
        # The same in the library's tiled order: 16 rows x 128 k a tile.
        rows, kt = -(-N // 16) * 16, -(-K // 128)
        full = torch.full((rows, kt * 128), 8, dtype=torch.uint8, device="cuda")
        full[:N, :K] = q
        v = full.view(rows // 16, 2, 8, kt, 4, 4, 8).permute(0, 3, 1, 2, 5, 4, 6)[..., list(NIBBLES)]
        s["tiled"] = (v[..., 0::2] | (v[..., 1::2] << 4)).contiguous().view(-1)
        per = 128 // group
        fs = torch.zeros(rows, kt * per, dtype=torch.bfloat16, device="cuda")
        fs[:N, :groups] = sc
        s["tiled_scales"] = fs.view(rows // 16, 16, kt, per).permute(0, 2, 1, 3).contiguous().view(-1)
        s["y"] = torch.empty(M, N, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms (32 bits)
def _scan(A, B):
    """All prefixes of h -> A h + B along the first axis, doubling the distance."""
    d = 1
    while d < A.shape[0]:
        B = torch.cat([B[:d], A[d:] * B[:-d] + B[d:]])
        A = torch.cat([A[:d], A[d:] * A[:-d]])
        d *= 2
    return B


def _gates(g, lengths):
    T, _, H2 = g.shape
    z = torch.sigmoid(g[..., : H2 // 2].float())
    n = g[..., H2 // 2:].float()
    if lengths is None:
        return z, n, None
    live = torch.arange(T, device=g.device)[:, None, None] < lengths[None, :, None]
    return torch.where(live, z, 1.0), torch.where(live, n, 0.0), live


def _recurrence(g, h0, lengths, h_type):
    z, n, live = _gates(g, lengths)
    b = (1.0 - z) * n
    b[0] += z[0] * h0
    h = _scan(z, b)
    last = h[-1].clone()
    if live is not None:
        h = torch.where(live, h, 0.0)
    return h.to(h_type), last


def _recurrence_backward(g, h0, lengths, h_out, dh_out, dh_last):
    z, n, live = _gates(g, lengths)
    dh = dh_out.float()
    if live is not None:
        dh = torch.where(live, dh, 0.0)
    e = z * dh
    e[-1] += z[-1] * dh_last
    e = _scan(z.flip(0), e.flip(0)).flip(0)  # e_t = z_t (dh_t + e_{t+1})
    d = dh + torch.cat([e[1:], dh_last[None]])
    before = torch.cat([h0[None], h_out[:-1].float()])
    dz = d * (before - n) * z * (1.0 - z)
    dn = d * (1.0 - z)
    if live is not None:
        dz, dn = torch.where(live, dz, 0.0), torch.where(live, dn, 0.0)
    return torch.cat([dz, dn], dim=-1).to(g.dtype), e[0]


def _step(g, slot_ids, state, h_type):
    H = state.shape[1]
    z = torch.sigmoid(g[:, :H].float())
    used = (slot_ids >= 0)[:, None]
    at = slot_ids.clamp(min=0).long()
    h = z * state[at] + (1.0 - z) * g[:, H:].float()
    new = torch.cat([state, state[:1]])  # a last row takes what padding rows write
    new[torch.where(used[:, 0], at, state.shape[0])] = h
    return torch.where(used, h, 0.0).to(h_type), new[:-1]


def _act(a, act):
    """The activation and its derivative."""
    if act == "relu":
        return torch.clamp(a, min=0.0), (a > 0).to(a.dtype)
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(a / math.sqrt(2.0)))
        return a * p, p + a * torch.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    s = torch.sigmoid(a)
    if act == "sigmoid":
        return s, s * (1.0 - s)
    return a * s, s * (1.0 + a * (1.0 - s))


def _glu(x, W, act):
    p = x @ W.T
    F = W.shape[0] // 2
    return _act(p[:, :F], act)[0] * p[:, F:]


def _glu_backward(x, W, dh, act):
    p = x @ W.T
    F = W.shape[0] // 2
    a, da = _act(p[:, :F], act)
    d = torch.cat([dh * p[:, F:] * da, dh * a], dim=1)
    return d @ W, d.T @ x


def _dequantised(codes, scales, group):
    q = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(1)
    return (q.to(torch.float32) - 8.0) * scales.float().repeat_interleave(group, dim=1)[:, : q.shape[1]]


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_1810_09958_gb300 import isam
        if op == "step":
            isam.glr_step(case["batch"], case["hidden"], case["slots"], s["g"], s["slot_ids"], s["state"],
                          s["new_state"], s["h"])
            return s["h"], s["new_state"]
        if op == "rfwd":
            isam.glr_forward(case["T"], case["batch"], case["hidden"], s["g"], s["h0"], s["lengths"], s["h_out"],
                             s["h_last"])
            return s["h_out"], s["h_last"]
        if op == "rbwd":
            isam.glr_backward(case["T"], case["batch"], case["hidden"], s["g"], s["h0"], s["lengths"], s["h_out"],
                              s["dh_out"], s["dh_last"], s["dg"], s["dh0"])
            return s["dg"], s["dh0"]
        if op == "gfwd":
            isam.glu_forward(case["T"], case["D"], case["F"], case["act"], s["x"], s["W"], s["h"])
            return s["h"]
        if op == "gbwd":
            isam.glu_backward(case["T"], case["D"], case["F"], case["act"], s["x"], s["W"], s["dh"], s["dx"], s["dW"])
            return s["dx"], s["dW"]
        isam.gemv_w4(case["M"], case["N"], case["K"], case["group"], s["x"], s["tiled"], s["tiled_scales"], s["y"])
        return s["y"]
    if op == "step":
        return _step(s["g"], s["slot_ids"], s["state"], s["h"].dtype)
    if op == "rfwd":
        return _recurrence(s["g"], s["h0"], s["lengths"], s["h_out"].dtype)
    if op == "rbwd":
        return _recurrence_backward(s["g"], s["h0"], s["lengths"], s["h_out"], s["dh_out"], s["dh_last"])
    if op == "gfwd":
        return _glu(s["x"].float(), s["W"].float(), case["act"]).bfloat16()
    if op == "gbwd":
        dx, dW = _glu_backward(s["x"].float(), s["W"].float(), s["dh"].float(), case["act"])
        return dx.bfloat16(), dW.bfloat16()
    return s["x"].float() @ _dequantised(s["codes"], s["scales"], case["group"]).T


def work(case):
    op = case["op"]
    size = {"bf16": 2, "fp32": 4}
    if op == "step":
        n = case["batch"] * case["hidden"]
        return dict(bytes=n * (2 * size[case["g"]] + 8 + size[case["h"]]) + 4 * case["batch"], flops=8.0 * n)
    if op in ("rfwd", "rbwd"):
        # A padded batch reads its live steps alone, and writes the zeros of the others too.
        n = case["T"] * case["batch"] * case["hidden"]
        live = sum(_lengths(case)) * case["hidden"] if case["ragged"] else n
        edge = case["batch"] * case["hidden"] * 4
        g, h = size[case["g"]], size[case["h"]]
        if op == "rfwd":
            return dict(bytes=live * 2 * g + n * h + 2 * edge, flops=10.0 * live)
        return dict(bytes=live * 2 * (g + h) + n * 2 * g + 3 * edge, flops=20.0 * live)
    if op in ("gfwd", "gbwd"):
        T, D, F = case["T"], case["D"], case["F"]
        if op == "gfwd":
            return dict(bytes=2.0 * (T * D + 2 * F * D + T * F), flops=4.0 * T * D * F)
        return dict(bytes=2.0 * (2 * T * D + 4 * F * D + T * F), flops=12.0 * T * D * F)
    M, N, K = case["M"], case["N"], case["K"]
    return dict(bytes=N * K / 2 + 2.0 * N * -(-K // case["group"]) + 2.0 * M * K + 4.0 * M * N, flops=2.0 * M * N * K)


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The definitions, step by step, in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "step":
        H = case["hidden"]
        g, state = s["g"].double(), s["state"].double()
        h = torch.zeros(case["batch"], H, dtype=torch.float64, device="cuda")
        for i, slot in enumerate(s["slot_ids"].tolist()):
            if slot >= 0:
                z = 1 / (1 + torch.exp(-g[i, :H]))
                h[i] = z * state[slot] + (1 - z) * g[i, H:]
                state[slot] = h[i]
        return h, state
    if op in ("rfwd", "rbwd"):
        T, B, H = case["T"], case["batch"], case["hidden"]
        live = torch.ones(T, B, 1, dtype=torch.bool, device="cuda")
        if s["lengths"] is not None:
            live = torch.arange(T, device="cuda")[:, None, None] < s["lengths"][:, None]
        gz, n = s["g"].double().masked_fill(~live, 0.0).split(H, dim=2)
        z = (1 / (1 + torch.exp(-gz))).masked_fill(~live, 1.0)  # padding keeps the state
        if op == "rfwd":
            h, out = s["h0"].double(), (1 - z) * n
            for t in range(T):
                h = out[t].addcmul_(z[t], h)
            return out.masked_fill(~live, 0.0), h
        d = s["dh_out"].double().masked_fill(~live, 0.0)
        e = s["dh_last"].double()
        for t in range(T - 1, -1, -1):
            d[t] += e
            e = z[t] * d[t]
        before = torch.cat([s["h0"].double()[None], s["h_out"][:-1].double()])
        dg = torch.cat([d * (before - n) * z * (1 - z), d * (1 - z)], dim=2)
        return dg.masked_fill(~live, 0.0), e
    if op in ("gfwd", "gbwd"):
        F, act = case["F"], case["act"]
        x, W = s["x"].double(), s["W"].double()
        gate, up = x @ W[:F].T, x @ W[F:].T
        t = torch.erf(gate * math.sqrt(0.5)) if act == "gelu" else 1 / (1 + torch.exp(-gate))
        if act == "silu":
            a, da = gate * t, t + gate * t * (1 - t)
        elif act == "gelu":
            a = gate * (1 + t) / 2
            da = (1 + t) / 2 + gate * torch.exp(-gate.square() / 2) / math.sqrt(2 * math.pi)
        elif act == "relu":
            a, da = gate.clamp(min=0), (gate > 0).double()
        else:
            a, da = t, t * (1 - t)
        if op == "gfwd":
            return a * up
        dh = s["dh"].double()
        dgate, dup = dh * up * da, dh * a
        return dgate @ W[:F] + dup @ W[F:], torch.cat([dgate.T @ x, dup.T @ x])
    K, group = case["K"], case["group"]
    y = torch.zeros(case["M"], case["N"], dtype=torch.float64, device="cuda")
    x = s["x"].double()
    for j in range(0, K, group):
        c = s["codes"][:, j // 2: min(j + group, K) // 2]
        w = torch.empty(c.shape[0], 2 * c.shape[1], dtype=torch.float64, device="cuda")
        w[:, 0::2] = (c % 16).double() - 8
        w[:, 1::2] = (c // 16).double() - 8
        y += (x[:, j: j + group] @ w.T) * s["scales"][:, j // group].double()
    return y
