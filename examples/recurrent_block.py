"""A recurrent language-model block trained and served with the library.

The block mixes over time with the gated linear recurrence and over features
with a gated feed-forward product, each around a residual:

    g  = x Wg^T            (isam_gemm, fp32)       z and n of the recurrence
    s  = recurrence(g)     (isam_glr_forward)      bf16 states
    x1 = x + s Wo^T        (isam_gemm)
    f  = silu(x1 Wf_gate^T) * (x1 Wf_up^T)         (isam_glu_forward)
    y  = x1 + f Wd^T       (isam_gemm)

``train`` takes steps of plain gradient descent on a synthetic target, the
gradients by isam_glu_backward, isam_glr_backward and isam_gemm.  ``serve``
packs the square projections to 4 bits (isam_w4_pack) and generates token by
token from a cache of states (isam_gemv_w4, isam_glr_step, isam_glu_forward),
then compares with the whole sequence at once on the same weights.

Run on a GB300 with the library built:  python examples/recurrent_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1810_09958_gb300 import isam  # noqa: E402

ACT, GROUP = "silu", 64


def gemm(A, B, transA=0, transB=0):
    """op(A) op(B), bf16 operands, fp32 result."""
    M, K = (A.shape[1], A.shape[0]) if transA else A.shape
    N = B.shape[0] if transB else B.shape[1]
    C = torch.empty(M, N, device=A.device)
    isam.gemm(M, N, K, transA, transB, 1.0, A, B, 0.0, C)
    return C


def bf16(x):
    return x.to(torch.bfloat16)


class Block:
    """Weights: Wg [2H][D] (z rows, n rows), Wo [D][H], Wf [2F][D] (gate rows, up rows), Wd [D][F]."""

    def __init__(self, D, H, F, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda n, k: bf16(torch.randn(n, k, generator=gen, device="cuda") / k ** 0.5)
        self.D, self.H, self.F = D, H, F
        self.W = dict(Wg=w(2 * H, D), Wo=w(D, H), Wf=w(2 * F, D), Wd=w(D, F))

    def forward(self, x, state):
        """x [T][B][D] bf16, state [B][H] fp32; returns y, the last state and what backward needs."""
        T, B, D = x.shape
        H, F, W = self.H, self.F, self.W
        xs = x.view(T * B, D)
        g = gemm(xs, W["Wg"], transB=1)
        s = torch.empty(T, B, H, dtype=torch.bfloat16, device=x.device)
        last = torch.empty(B, H, device=x.device)
        isam.glr_forward(T, B, H, g, state, None, s, last)
        x1 = bf16(xs + gemm(s.view(T * B, H), W["Wo"], transB=1))
        f = torch.empty(T * B, F, dtype=torch.bfloat16, device=x.device)
        isam.glu_forward(T * B, D, F, ACT, x1, W["Wf"], f)
        y = x1 + gemm(f, W["Wd"], transB=1)
        return y.view(T, B, D), last, (xs, g, state, s, x1, f)

    def backward(self, dy, kept):
        """Gradients of every weight from dy [T][B][D]."""
        xs, g, state, s, x1, f = kept
        T, B, H = s.shape
        D, F, W = self.D, self.F, self.W
        dyb = bf16(dy.view(T * B, D))
        d = dict(Wd=gemm(dyb, f, transA=1), Wf=torch.empty_like(W["Wf"]))
        dx1 = torch.empty_like(x1)
        isam.glu_backward(T * B, D, F, ACT, x1, W["Wf"], bf16(gemm(dyb, W["Wd"])), dx1, d["Wf"])
        dx1 = bf16(dx1 + dy.view(T * B, D))
        s2 = s.view(T * B, H)
        d["Wo"] = gemm(dx1, s2, transA=1)
        dg = torch.empty_like(g)
        isam.glr_backward(T, B, H, g, state, None, s, bf16(gemm(dx1, W["Wo"])), None, dg)
        d["Wg"] = gemm(bf16(dg), xs, transA=1)
        return d


def train(D=512, H=512, F=1024, T=64, B=4, steps=30, rate=0.3):
    """Losses of a few steps towards a fixed target: each token's running mean of the inputs so far."""
    block = Block(D, H, F)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = bf16(torch.randn(T, B, D, generator=gen, device="cuda"))
    want = x.float().cumsum(0) / torch.arange(1, T + 1, device="cuda").view(T, 1, 1)
    master = {k: v.float() for k, v in block.W.items()}
    state = torch.zeros(B, H, device="cuda")
    losses = []
    for _ in range(steps):
        y, _, kept = block.forward(x, state)
        err = y - want
        losses.append(float(err.square().mean()))
        for k, d in block.backward(err * (2.0 / (T * B)), kept).items():
            master[k] -= rate / D ** 0.5 * d.float()
            block.W[k] = bf16(master[k])
    isam.sync()
    return block, losses


def quantise(W):
    """Rows in groups of GROUP: codes (two a byte), scales, and the weights that they stand for."""
    N, K = W.shape
    v = W.float().view(N, K // GROUP, GROUP)
    scale = bf16(v.abs().amax(2, keepdim=True) / 7.0).clamp_(min=1e-8)
    q = (v / scale.float()).round().clamp(-8, 7)
    back = bf16((q * scale.float()).view(N, K))
    q = (q.view(N, K) + 8).to(torch.uint8)
    return q[:, 0::2] | (q[:, 1::2] << 4), scale.view(N, K // GROUP), back


class Packed:
    def __init__(self, W):
        self.N, self.K = W.shape
        codes, scales, self.dense = quantise(W)
        self.tiled = torch.empty(isam.w4_tiled_bytes(self.N, self.K), dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(isam.w4_tiled_scales(self.N, self.K, GROUP), dtype=torch.bfloat16, device="cuda")
        isam.w4_pack(self.N, self.K, GROUP, codes.contiguous(), scales.contiguous(), self.tiled, self.scales)

    def __call__(self, x):
        y = torch.empty(x.shape[0], self.N, device="cuda")
        isam.gemv_w4(x.shape[0], self.N, self.K, GROUP, x, self.tiled, self.scales, y)
        return y


def serve(block, T=24, B=3, slots=8):
    """Token by token with 4-bit projections against the whole sequence: the largest difference over the largest output."""
    D, H, F = block.D, block.H, block.F
    packed = {k: Packed(block.W[k]) for k in ("Wg", "Wo", "Wd")}
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = bf16(torch.randn(T, B, D, generator=gen, device="cuda"))
    cache = torch.zeros(slots, H, device="cuda")
    ids = torch.tensor([5, 0, 6], dtype=torch.int32, device="cuda")[:B]
    out = torch.empty(T, B, D, device="cuda")
    s = torch.empty(B, H, dtype=torch.bfloat16, device="cuda")
    f = torch.empty(B, F, dtype=torch.bfloat16, device="cuda")
    for t in range(T):
        isam.glr_step(B, H, slots, packed["Wg"](x[t]), ids, cache, cache, s)
        x1 = bf16(x[t] + packed["Wo"](s))
        isam.glu_forward(B, D, F, ACT, x1, block.W["Wf"], f)
        out[t] = x1 + packed["Wd"](f)
    dense = Block(D, H, F)
    dense.W = dict(block.W, **{k: p.dense for k, p in packed.items()})
    whole, last, _ = dense.forward(x, torch.zeros(B, H, device="cuda"))
    isam.sync()
    scale = float(whole.abs().max())
    return float((out - whole).abs().max()) / scale, float((cache[ids.long()] - last).abs().max())


if __name__ == "__main__":
    trained, losses = train()
    print("loss of each step:", " ".join("%.3f" % v for v in losses))
    print("serving against the whole sequence: outputs %.2g, states %.2g" % serve(trained))
