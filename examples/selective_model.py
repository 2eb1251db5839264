"""A small selective state space model served with the library: prompts at once,
then beam search a token at a time.

A layer mixes over time with a short convolution and the selective scan, behind
a norm whose output goes to a block-scaled product:

    r      = r + x;  n = norm(r)                       (isam_rms_norm_forward, E4M3 and scales)
    x | z  = n Win^T                                   (isam_gemm_mxfp8, fp32)
    u      = silu(conv(x))                             (isam_conv1d_forward / isam_conv1d_step)
    dt' | B | C = u Wx^T;  dt = dt' Wdt^T              (isam_gemm)
    y      = scan(u, dt, A, B, C) silu(z)              (isam_ssm_forward / isam_ssm_step)
    x      = y Wout^T                                  (isam_gemm)

The last norm's output times the embedding gives the logits.  ``search`` runs
prompts and then picks the best continuations step by step (isam_beam_select);
the layers' states follow the chosen beams (isam_beam_reorder).

Run on a GB300 with the library built:  python examples/selective_model.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1810_09958_gb300 import isam  # noqa: E402

EPS, WIDTH = 1e-5, 4


def gemm(x, W):
    """x W^T, bf16 operands, fp32 result."""
    y = torch.empty(x.shape[0], W.shape[0], device=x.device)
    isam.gemm(x.shape[0], W.shape[0], x.shape[1], 0, 1, 1.0, x, W, 0.0, y)
    return y


def block_scaled(W):
    """A weight's E4M3 bytes and scales (a norm whose rows come out as they went in)."""
    N, K = W.shape
    size = W.float().square().mean(dim=1, keepdim=True).sqrt()
    q = torch.empty(N, K, dtype=torch.uint8, device=W.device)
    s = torch.empty(-(-K // 128), N, 4, dtype=torch.uint8, device=W.device)
    isam.rms_norm_forward(N, K, (W.float() / size).contiguous(), None, None, torch.ones(K, device=W.device), 0.0, None, q, s)
    return q, s, size


class Model:
    def __init__(self, V=512, D=128, C=256, N=16, R=8, layers=2, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
        self.V, self.D, self.C, self.N, self.R = V, D, C, N, R
        self.embed = normal(V, D).bfloat16()
        self.norm = torch.ones(D, device="cuda")
        self.layers = []
        for _ in range(layers):
            Win = normal(2 * C, D) / D ** 0.5
            q, s, size = block_scaled(Win)
            self.layers.append(dict(
                norm=1.0 + 0.1 * normal(D), Win=q, Win_scales=s, Win_size=size.view(-1).contiguous(),
                conv=normal(WIDTH, C) / WIDTH ** 0.5, conv_bias=0.1 * normal(C),
                Wx=(normal(R + 2 * N, C) / C ** 0.5).bfloat16(), Wdt=(normal(C, R) / R ** 0.5).bfloat16(),
                dt_bias=normal(C) - 3.0, A=-torch.arange(1, N + 1, device="cuda", dtype=torch.float32).repeat(C, 1),
                D=normal(C), Wout=(normal(D, C) / C ** 0.5).bfloat16()))

    def states(self, slots):
        """Caches of all layers: the convolutions' last inputs, the scans' states."""
        n = len(self.layers)
        return (torch.zeros(n, slots, WIDTH - 1, self.C, device="cuda"), torch.zeros(n, slots, self.C, self.N, device="cuda"))

    def forward(self, tokens, states, lengths=None, slot_ids=None):
        """Logits [rows][V] of tokens [T][batch] (whole sequences, padded behind `lengths`), or of [batch] (one
        more token each, states in rows slot_ids).  The states are updated in place."""
        C, D, N, R = self.C, self.D, self.N, self.R
        whole = tokens.dim() == 2
        T, batch = tokens.shape if whole else (1, tokens.shape[0])
        rows, slots = T * batch, states[0].shape[1]
        x, r = torch.zeros(rows, D, device="cuda"), self.embed[tokens.view(-1)].float()
        n8 = torch.empty(rows, D, dtype=torch.uint8, device="cuda")
        scales = torch.empty(-(-D // 128), rows, 4, dtype=torch.uint8, device="cuda")
        xz = torch.empty(rows, 2 * C, device="cuda")
        u, y = (torch.empty(rows, C, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for layer, conv, scan in zip(self.layers, *states):
            isam.rms_norm_forward(rows, D, x, r, r, layer["norm"], EPS, None, n8, scales)
            isam.gemm_mxfp8(rows, 2 * C, D, 1.0, n8, scales, layer["Win"], layer["Win_scales"], 0.0, xz)
            xz *= layer["Win_size"]
            if whole:
                isam.conv1d_forward(T, batch, C, WIDTH, xz[:, :C], layer["conv"], layer["conv_bias"], True, conv[:batch],
                                    lengths, u, conv[:batch])
            else:
                isam.conv1d_step(batch, C, WIDTH, slots, xz[:, :C], layer["conv"], layer["conv_bias"], True, slot_ids, conv,
                                 conv, u)
            p = gemm(u, layer["Wx"])
            dt = gemm(p[:, :R].bfloat16(), layer["Wdt"])
            args = (u, dt, layer["dt_bias"], layer["A"], p[:, R: R + N], p[:, R + N:], layer["D"], xz[:, C:])
            if whole:
                isam.ssm_forward(T, batch, C, N, *args, scan[:batch], lengths, y, scan[:batch])
            else:
                isam.ssm_step(batch, C, N, slots, *args, slot_ids, scan, scan, y)
            x = gemm(y, layer["Wout"])
        n = torch.empty(rows, D, dtype=torch.bfloat16, device="cuda")
        isam.rms_norm_forward(rows, D, x, r, None, self.norm, EPS, n)
        return gemm(n, self.embed) / D ** 0.5


def search(model, prompts, lengths, steps, beams=4, eos=0):
    """Beam search behind prompts [T][batch] (padded): tokens [batch][beams][steps] and scores [batch][beams], best first."""
    T, batch = prompts.shape
    states = model.states(batch * beams)
    logits = model.forward(prompts, states, lengths).view(T, batch, -1)
    last = logits[lengths.long() - 1, torch.arange(batch, device="cuda")]
    # The prompt's states go to its sequence's first beam, and from there to all.
    first = torch.arange(batch, device="cuda") * beams
    for cache in states:
        cache[:, first] = cache[:, :batch].clone()
    scores = torch.full((batch, beams), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    new = lambda kind: torch.empty(batch, beams, dtype=kind, device="cuda")
    parents, tokens, ended = new(torch.int32), new(torch.int32), torch.zeros(batch, beams, dtype=torch.bool, device="cuda")
    out = torch.zeros(batch, beams, 0, dtype=torch.int32, device="cuda")
    logits = last[:, None].expand(batch, beams, model.V).contiguous()
    for _ in range(steps):
        isam.beam_select(batch, beams, model.V, beams, logits, scores, eos, ended, scores, parents, tokens, ended)
        out = torch.cat([torch.gather(out, 1, parents.long()[..., None].expand_as(out)), tokens[..., None]], dim=2)
        for cache in states:
            isam.beam_reorder(len(model.layers), batch, beams, batch * beams, parents, None, cache, cache)
        logits = model.forward(tokens.view(-1).long(), states).view(batch, beams, model.V)
    isam.sync()
    return out, scores


if __name__ == "__main__":
    model = Model()
    gen = torch.Generator(device="cuda").manual_seed(1)
    found, scores = search(model, torch.randint(1, model.V, (24, 3), generator=gen, device="cuda"),
                           torch.tensor([24, 1, 17], dtype=torch.int32, device="cuda"), 8)
    for b in range(3):
        print("sequence %d:" % b, " | ".join("%s (%.2f)" % (t.tolist(), s) for t, s in zip(found[b], scores[b])))
