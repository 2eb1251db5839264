"""The example that runs the norm, the block-scaled product, the convolution, the
scan and beam search together, against the same model in 64 bits; and a
trained block of norm and feed-forward product, whose gradients are autograd's."""
import os
import sys

import numpy as np
import pytest
import torch

import serve_ref as ref

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example():
    import selective_model
    return selective_model


def values(q, s):
    """What block-scaled bytes stand for."""
    N, K = q.shape
    byte = s.cpu().numpy().transpose(1, 0, 2).reshape(N, -1).astype(np.int64)
    return ref.e4m3(q.cpu().numpy()) * np.repeat(2.0 ** (byte - 127.0), 32, axis=1)[:, :K]


class Plain:
    """The model in numpy, 64 bits, its weights as the library holds them (nothing rounded in between)."""

    def __init__(self, m, width):
        self.m, self.width = m, width
        f = lambda t: t.double().cpu().numpy()
        self.embed, self.norm = f(m.embed), f(m.norm)
        self.layers = [{k: f(v) for k, v in l.items() if k not in ("Win", "Win_scales")} |
                       dict(Win=values(l["Win"], l["Win_scales"]) * f(l["Win_size"])[:, None]) for l in m.layers]

    def logits(self, tokens):
        """tokens [T] of one sequence -> [T][V]."""
        m, T = self.m, len(tokens)
        C, N, R = m.C, m.N, m.R
        x, r = 0.0, self.embed[tokens]
        for l in self.layers:
            n, r = ref.norm(r, x, l["norm"], 1e-5)
            xz = n @ l["Win"].T
            u, _, _ = ref.conv(xz[:, None, :C], l["conv"], l["conv_bias"], True, np.zeros((1, self.width - 1, C)), [T])
            p = u[:, 0] @ l["Wx"].T
            dt = p[:, :R] @ l["Wdt"].T
            y, _, _, _ = ref.scan(u, dt[:, None], l["dt_bias"], l["A"], p[:, None, R: R + N], p[:, None, R + N:], l["D"],
                                  xz[:, None, C:], np.zeros((1, C, N)), np.array([T]), "fp32")
            x = y[:, 0] @ l["Wout"].T
        n, _ = ref.norm(r, x, self.norm, 1e-5)
        return n @ self.embed.T / m.D ** 0.5


def near(got, want):
    """Norms agree to 6%: a layer rounds its norm's output to E4M3 (2^-4 of a value at most, 2.6% in the mean
    square) and three more values to bf16; two layers' errors add up as squares, and the scan's gates about double them."""
    return np.linalg.norm(got - want) <= 0.06 * np.linalg.norm(want)


def test_prompts_and_tokens_are_the_plain_models(example):
    m = example.Model(seed=3)
    plain = Plain(m, example.WIDTH)
    T, batch, more = 13, 3, 4
    lengths = np.array([13, 1, 8])
    gen = torch.Generator(device="cuda").manual_seed(4)
    tokens = torch.randint(0, m.V, (T + more, batch), generator=gen, device="cuda")
    states = m.states(5)
    logits = m.forward(tokens[:T], states, torch.from_numpy(lengths).int().cuda()).view(T, batch, -1).double().cpu().numpy()
    for b, n in enumerate(lengths):
        line = tokens[:n, b].cpu().numpy()
        assert near(logits[:n, b], plain.logits(line))
        for i in range(more):  # one token at a time, the others' states in use meanwhile
            ids = torch.full((batch,), -1, dtype=torch.int32, device="cuda")
            ids[b] = b
            out = m.forward(tokens[T + i], states, slot_ids=ids).double().cpu().numpy()
            line = np.append(line, tokens[T + i, b].item())
            assert near(out[b], plain.logits(line)[-1])


def test_search_scores_are_its_sequences(example):
    """Every beam's score is the sum of its tokens' log-probabilities in the plain model, up to what the model's own
    rounding moves them (near() on logits of norm sqrt(V): at most 0.06 each where they are independent; 0.3
    a token is allowed), beams are distinct and in order, and an ended beam stays."""
    m = example.Model(seed=5)
    plain = Plain(m, example.WIDTH)
    gen = torch.Generator(device="cuda").manual_seed(6)
    prompts, lengths = torch.randint(1, m.V, (9, 2), generator=gen, device="cuda"), [9, 4]
    steps, eos = 5, 7
    m.embed[eos] *= 2.5  # an end that comes up
    plain = Plain(m, example.WIDTH)
    found, scores = example.search(m, prompts, torch.tensor(lengths, dtype=torch.int32, device="cuda"), steps, 4, eos)
    for b in range(2):
        seen = set()
        assert (scores[b].diff() <= 0).all()
        for k in range(4):
            line = found[b, k].tolist()
            assert tuple(line) not in seen
            seen.add(tuple(line))
            stop = line.index(eos) + 1 if eos in line else steps
            assert line[stop:] == [eos] * (steps - stop)
            whole = np.concatenate([prompts[:lengths[b], b].cpu().numpy(), line[:stop]])
            logits = plain.logits(whole)
            total = 0.0
            for i in range(stop):
                row = logits[lengths[b] - 1 + i]
                total += row[line[i]] - row.max() - np.log(np.exp(row - row.max()).sum())
            assert abs(scores[b, k].item() - total) <= 0.3 * stop


def test_norm_and_feed_forward_gradients_are_autograds():
    """y = x + glu(norm(x)) and its gradients: four values are rounded to bf16 between a weight and the loss; 3% as
    for the recurrent block."""
    from paper_1810_09958_gb300 import isam
    T, D, F = 96, 128, 160
    gen = torch.Generator(device="cuda").manual_seed(7)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, w = normal(T, D).bfloat16(), 1 + 0.2 * normal(D)
    W, dh = (normal(2 * F, D) / D ** 0.5).bfloat16(), normal(T, F).bfloat16()
    n, h = torch.empty_like(x), torch.empty(T, F, dtype=torch.bfloat16, device="cuda")
    dn, dW, dx, dw = torch.empty_like(x), torch.empty_like(W), torch.empty_like(x), torch.empty(D, device="cuda")
    dres = normal(T, D).bfloat16()
    isam.rms_norm_forward(T, D, x, None, None, w, 1e-5, n)
    isam.glu_forward(T, D, F, "silu", n, W, h)
    isam.glu_backward(T, D, F, "silu", n, W, dh, dn, dW)
    isam.rms_norm_backward(T, D, x, w, 1e-5, dn, dres, dx, dw)
    isam.sync()
    xd, wd, Wd = x.double().requires_grad_(), w.double().requires_grad_(), W.double().requires_grad_()
    nd = xd / torch.sqrt(xd.square().mean(1, keepdim=True) + 1e-5) * wd
    p = nd @ Wd.T
    hd = torch.nn.functional.silu(p[:, :F]) * p[:, F:]
    ((hd * dh.double()).sum() + (xd * dres.double()).sum()).backward()
    for got, want in ((h, hd.detach()), (dx, xd.grad), (dw, wd.grad), (dW, Wd.grad)):
        assert (got.double() - want).norm() <= 0.03 * want.norm()
