"""Selective state space scan over a sequence and for one token, against the
definition in 64 bits."""
import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_1810_09958_gb300 import isam
from test_conv1d_gpu import close, rows
from test_norm_gpu import TYPES, guarded, intact, tensor

pytestmark = pytest.mark.gpu


class Operands:
    def __init__(self, seed, T, batch, C, N, u_kind="bf16", p_kind="fp32", gate=True, wide="last", bias=True, slow=False):
        rng = np.random.default_rng(seed)
        shape = (T, batch) if T else (batch,)
        self.u, self.u64 = tensor(rng, (*shape, C), u_kind)
        self.dt, self.dt64 = tensor(rng, (*shape, C), p_kind)
        self.bias, self.bias64 = tensor(rng, (C,), "fp32")
        if slow:  # steps that keep nearly all of the state
            self.bias -= 6.0
            self.bias64 = self.bias.double().cpu().numpy()
        if not bias:
            self.bias, self.bias64 = None, np.zeros(C)
        A = -np.exp(rng.uniform(-3, 2.5, (C, N))).astype(np.float32)
        self.A, self.A64 = torch.from_numpy(A).cuda(), A.astype(np.float64)
        bc, bc64 = tensor(rng, (*shape, 2 * N + 5), p_kind)
        self.B, self.Cm, self.B64, self.C64 = bc[..., :N], bc[..., N: 2 * N], bc64[..., :N], bc64[..., N: 2 * N]
        self.D, self.D64 = tensor(rng, (C,), "fp32")
        self.z, self.z64 = rows(rng, (*shape, C), p_kind, wide) if gate else (None, None)
        self.h0, self.h064 = tensor(rng, (batch, C, N), "fp32")
        self.kind = u_kind

    def ref(self, lengths, h0=None):
        z = self.z64
        return ref.scan(self.u64, self.dt64, self.bias64, self.A64, self.B64, self.C64, self.D64, z,
                        self.h064 if h0 is None else h0, lengths, self.kind)


SHAPES = [(1, 1, 1, 1), (1, 3, 40, 16), (2, 2, 33, 7), (5, 1, 64, 16), (17, 2, 100, 12), (64, 1, 8, 16), (100, 3, 65, 16),
          (256, 1, 16, 8), (777, 2, 9, 16), (300, 1, 12, 20), (130, 1, 5, 64), (65, 2, 3, 100), (40, 1, 6, 128),
          (1500, 1, 3, 3), (33, 40, 32, 16), (9, 1, 1000, 16), (129, 1, 128, 16), (515, 1, 34, 16)]


@pytest.mark.parametrize("u_kind,p_kind,gate,wide", [("bf16", "fp32", True, "last"), ("fp32", "bf16", False, "no"),
                                                     ("fp32", "fp32", True, "odd"), ("bf16", "bf16", True, "no")])
@pytest.mark.parametrize("T,batch,C,N", SHAPES)
def test_forward(T, batch, C, N, u_kind, p_kind, gate, wide):
    o = Operands(T * 1000 + C, T, batch, C, N, u_kind, p_kind, gate, wide, slow=T % 2 == 1)
    whole, y = guarded(T * batch * C, TYPES[u_kind])
    whole_h, last = guarded(batch * C * N, torch.float32)
    isam.ssm_forward(T, batch, C, N, o.u, o.dt, o.bias, o.A, o.B, o.Cm, o.D, o.z, o.h0, None, y, last)
    isam.sync()
    want, h, ey, eh = o.ref(np.full(batch, T))
    assert close(y.view(T, batch, C), want, ey)
    assert close(last.view(batch, C, N), h, eh)
    assert intact(whole, T * batch * C) and intact(whole_h, batch * C * N)


@pytest.mark.parametrize("C,N", [(48, 16), (33, 5), (7, 40), (130, 16)])
@pytest.mark.parametrize("in_place", [False, True])
def test_padded_batch(C, N, in_place):
    """Lengths of zero and one, beyond T and below zero, NaN and infinities in padding, no bias, no D."""
    T = 290
    lengths = np.array([290, 0, 1, 64, 65, 128, 999, -5])
    batch = len(lengths)
    o = Operands(C, T, batch, C, N, "fp32", "fp32", True, "last", bias=False)
    n = lengths.clip(0, T)
    pad = torch.from_numpy(np.arange(T)[:, None] >= n[None]).cuda()
    for t, v in ((o.u, "nan"), (o.dt, "inf"), (o.B, "nan"), (o.Cm, "-inf"), (o.z, "nan")):
        t[pad] = float(v)
    y = torch.full((T, batch, C), 9.0, device="cuda")
    last = o.h0 if in_place else torch.empty_like(o.h0)
    isam.ssm_forward(T, batch, C, N, o.u, o.dt, None, o.A, o.B, o.Cm, None, o.z, o.h0, torch.from_numpy(lengths).int().cuda(),
                     y, last)
    isam.sync()
    o.D64 = np.zeros(C)
    want, h, ey, eh = o.ref(n)
    assert close(y, want, ey) and close(last, h, eh)
    assert not y[pad].any()


def test_without_states_and_z():
    T, batch, C, N = 50, 2, 24, 16
    o = Operands(3, T, batch, C, N, "fp32", "fp32", False)
    y = torch.empty(T, batch, C, device="cuda")
    isam.ssm_forward(T, batch, C, N, o.u, o.dt, o.bias, o.A, o.B, o.Cm, o.D, None, None, None, y)
    want, _, ey, _ = o.ref(np.full(batch, T), np.zeros((batch, C, N)))
    assert close(y, want, ey)


def test_extreme_steps():
    """delta of 1e-6 (softplus far below zero) to 50, decays that underflow, growing states."""
    T, batch, C, N = 120, 1, 64, 16
    o = Operands(4, T, batch, C, N, "fp32", "fp32", False)
    shift = torch.linspace(-14, 50, C, device="cuda")
    o.dt += shift
    o.dt64 = o.dt.double().cpu().numpy()
    o.A[::7] *= -0.0005  # states that grow a little
    o.A64 = o.A.double().cpu().numpy()
    y, last = torch.empty(T, batch, C, device="cuda"), torch.empty(batch, C, N, device="cuda")
    isam.ssm_forward(T, batch, C, N, o.u, o.dt, o.bias, o.A, o.B, o.Cm, o.D, None, o.h0, None, y, last)
    want, h, ey, eh = o.ref(np.full(batch, T))
    assert close(y, want, ey) and close(last, h, eh)


@pytest.mark.parametrize("u_kind,p_kind,gate,wide", [("bf16", "fp32", True, "last"), ("fp32", "bf16", False, "no"),
                                                     ("fp32", "fp32", True, "odd")])
@pytest.mark.parametrize("batch,C,N,in_place", [(1, 1, 1, False), (5, 64, 16, True), (33, 129, 12, False), (3, 40, 7, True),
                                                (2, 17, 20, False), (4, 9, 64, True), (2, 5, 128, False), (3, 6, 33, True),
                                                (70, 512, 16, True)])
def test_step(batch, C, N, in_place, u_kind, p_kind, gate, wide):
    o = Operands(batch * 1000 + C, 0, batch, C, N, u_kind, p_kind, gate, wide)
    slots = batch + 2
    rng = np.random.default_rng(C)
    ids = rng.permutation(slots)[:batch]
    if batch > 2:
        ids[1], ids[2] = -1, slots  # padding rows
    state, state64 = tensor(rng, (slots, C, N), "fp32")
    new = state if in_place else torch.full_like(state, 5.0)
    whole, y = guarded(batch * C, TYPES[u_kind])
    isam.ssm_step(batch, C, N, slots, o.u, o.dt, o.bias, o.A, o.B, o.Cm, o.D, o.z, torch.from_numpy(ids).int().cuda(),
                  state, new, y)
    isam.sync()
    left = state64.copy() if in_place else np.full_like(state64, 5.0)
    tol = np.zeros_like(left)
    want, ey = np.zeros((batch, C)), np.zeros((batch, C))
    for i, slot in enumerate(ids):
        if 0 <= slot < slots:
            z = None if o.z64 is None else o.z64[None, i: i + 1]
            v, h, e, eh = ref.scan(o.u64[None, i: i + 1], o.dt64[None, i: i + 1], o.bias64, o.A64, o.B64[None, i: i + 1],
                                   o.C64[None, i: i + 1], o.D64, z, state64[slot: slot + 1], np.ones(1), u_kind)
            want[i], ey[i], left[slot], tol[slot] = v[0, 0], e[0, 0], h[0], eh[0]
    assert close(y.view(batch, C), want, ey)
    assert close(new, left, tol)
    assert intact(whole, batch * C)


def test_tokens_after_a_prompt_are_the_longer_prompt():
    T, more, batch, C, N = 90, 5, 3, 64, 16
    o = Operands(9, T + more, batch, C, N, "fp32", "fp32")
    first, state = torch.empty(T, batch, C, device="cuda"), torch.empty(batch, C, N, device="cuda")
    isam.ssm_forward(T, batch, C, N, o.u[:T], o.dt[:T], o.bias, o.A, o.B[:T], o.Cm[:T], o.D, o.z[:T], o.h0, None, first, state)
    got = [first]
    for t in range(T, T + more):
        one = torch.empty(batch, C, device="cuda")
        isam.ssm_step(batch, C, N, batch, o.u[t], o.dt[t], o.bias, o.A, o.B[t], o.Cm[t], o.D, o.z[t], None, state, state, one)
        got.append(one[None])
    want, h, ey, eh = o.ref(np.full(batch, T + more))
    assert close(torch.cat(got), want, ey) and close(state, h, eh)


def test_the_same_call_twice_and_replayed():
    T, batch, C, N = 600, 1, 96, 16
    o = Operands(10, T, batch, C, N)
    out = [(torch.empty(T, batch, C, dtype=torch.bfloat16, device="cuda"), torch.empty(batch, C, N, device="cuda")) for _ in range(3)]

    def call(y, last):
        isam.ssm_forward(T, batch, C, N, o.u, o.dt, o.bias, o.A, o.B, o.Cm, o.D, o.z, o.h0, None, y, last)

    call(*out[0])
    call(*out[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*out[2])
    graph.replay()
    torch.cuda.synchronize()
    for y, last in out[1:]:
        assert torch.equal(y, out[0][0]) and torch.equal(last, out[0][1])


def test_on_another_stream():
    T, batch, C, N = 64, 2, 256, 16
    o = Operands(11, T, batch, C, N, "fp32")
    y, y2 = torch.empty(T, batch, C, device="cuda"), torch.zeros(T, batch, C, device="cuda")
    isam.ssm_forward(T, batch, C, N, o.u, o.dt, o.bias, o.A, o.B, o.Cm, o.D, o.z, o.h0, None, y)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        isam.ssm_forward(T, batch, C, N, o.u, o.dt, o.bias, o.A, o.B, o.Cm, o.D, o.z, o.h0, None, y2)
    side.synchronize()
    assert torch.equal(y, y2)
