"""Causal convolution over a sequence and for one token, against the
definition in 64 bits."""
import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_1810_09958_gb300 import isam
from test_norm_gpu import TYPES, guarded, intact, tensor

pytestmark = pytest.mark.gpu


def rows(rng, shape, kind, wide):
    """x as columns of wider rows (wide: the first or the last half, or rows 3 apart), and its values."""
    C = shape[-1]
    extra = {"no": 0, "first": C, "last": C, "odd": 3}[wide]
    t, v = tensor(rng, (*shape[:-1], C + extra), kind)
    return (t[..., C:], v[..., C:]) if wide == "last" else (t[..., :C], v[..., :C])


def close(got, want, bound):
    return bool((np.abs(got.double().cpu().numpy() - want) <= bound).all())


@pytest.mark.parametrize("x_kind,y_kind,wide,width,act", [
    ("bf16", "bf16", "no", 4, True), ("fp32", "bf16", "first", 4, True), ("bf16", "fp32", "last", 2, False),
    ("fp32", "fp32", "odd", 3, True), ("bf16", "bf16", "odd", 8, True), ("fp32", "bf16", "no", 5, False),
    ("fp32", "fp32", "no", 6, True), ("bf16", "fp32", "no", 7, True)])
@pytest.mark.parametrize("T,batch,C", [(1, 1, 1), (1, 3, 8), (2, 2, 64), (3, 1, 65), (7, 2, 128), (33, 5, 36), (64, 1, 512),
                                       (130, 2, 1000), (5, 70, 24), (300, 3, 4)])
def test_forward(T, batch, C, x_kind, y_kind, wide, width, act):
    rng = np.random.default_rng(T * 1000 + C)
    x, x64 = rows(rng, (T, batch, C), x_kind, wide)
    w, w64 = tensor(rng, (width, C), "fp32")
    bias, bias64 = tensor(rng, (C,), "fp32")
    state, state64 = tensor(rng, (batch, width - 1, C), x_kind)
    whole, y = guarded(T * batch * C, TYPES[y_kind])
    whole_s, new = guarded(batch * (width - 1) * C, TYPES[x_kind])
    isam.conv1d_forward(T, batch, C, width, x, w, bias, act, state, None, y, new)
    isam.sync()
    want, last, size = ref.conv(x64, w64, bias64, act, state64, np.full(batch, T))
    assert close(y.view(T, batch, C), want, ref.conv_bound(want, size, width, act, y_kind))
    assert close(new.view(batch, width - 1, C), last, 0.0)
    assert intact(whole, T * batch * C) and intact(whole_s, batch * (width - 1) * C)


@pytest.mark.parametrize("C", [40, 41])
@pytest.mark.parametrize("in_place", [False, True])
def test_padded_batch(C, in_place):
    """Lengths of zero and one, beyond T and below zero, NaN in padding, no bias, states of short sequences."""
    T, width = 70, 4
    lengths = np.array([70, 0, 1, 2, 3, 35, 999, -5, 64])
    batch = len(lengths)
    rng = np.random.default_rng(C)
    x, x64 = tensor(rng, (T, batch, C), "bf16")
    pad = np.arange(T)[:, None] >= lengths.clip(0, T)[None]
    x[torch.from_numpy(pad).cuda()] = float("nan")
    w, w64 = tensor(rng, (width, C), "fp32")
    state, state64 = tensor(rng, (batch, width - 1, C), "bf16")
    y = torch.full((T, batch, C), 9.0, device="cuda")
    new = state if in_place else torch.empty_like(state)
    isam.conv1d_forward(T, batch, C, width, x, w, None, True, state, torch.from_numpy(lengths).int().cuda(), y, new)
    isam.sync()
    want, last, size = ref.conv(np.where(pad[..., None], 0, x64), w64, np.zeros(C), True, state64, lengths)
    assert close(y, want, ref.conv_bound(want, size, width, True, "fp32"))
    assert close(new, last, 0.0)
    assert not y.cpu().numpy()[pad].any()


@pytest.mark.parametrize("width", [2, 5, 6, 8])
def test_states_in_place_of_every_width(width):
    """Few rows, thus short runs: none but a sequence's first may look at states that this one overwrites."""
    T, batch, C = 64, 2, 200
    rng = np.random.default_rng(width)
    x, _ = tensor(rng, (T, batch, C), "bf16")
    w, _ = tensor(rng, (width, C), "fp32")
    state, _ = tensor(rng, (batch, width - 1, C), "bf16")
    y, new = torch.empty_like(x), torch.empty_like(state)
    isam.conv1d_forward(T, batch, C, width, x, w, None, True, state, None, y, new)
    for _ in range(50):
        there, got = state.clone(), torch.empty_like(x)
        isam.conv1d_forward(T, batch, C, width, x, w, None, True, there, None, got, there)
        assert torch.equal(got, y) and torch.equal(there, new)


def test_without_states():
    T, batch, C = 9, 2, 16
    rng = np.random.default_rng(1)
    x, x64 = tensor(rng, (T, batch, C), "fp32")
    w, w64 = tensor(rng, (3, C), "fp32")
    y = torch.empty(T, batch, C, device="cuda")
    isam.conv1d_forward(T, batch, C, 3, x, w, None, False, None, None, y)
    want, _, size = ref.conv(x64, w64, np.zeros(C), False, np.zeros((batch, 2, C)), np.full(batch, T))
    assert close(y, want, ref.conv_bound(want, size, 3, False, "fp32"))


@pytest.mark.parametrize("x_kind,y_kind,wide,width", [("fp32", "bf16", "first", 4), ("bf16", "fp32", "odd", 3),
                                                      ("bf16", "bf16", "no", 2), ("fp32", "fp32", "last", 8)])
@pytest.mark.parametrize("batch,C,in_place", [(1, 1, False), (5, 64, True), (33, 129, False), (64, 1024, True)])
def test_step(batch, C, in_place, x_kind, y_kind, wide, width):
    rng = np.random.default_rng(batch * 1000 + C)
    slots = batch + 3
    x, x64 = rows(rng, (batch, C), x_kind, wide)
    w, w64 = tensor(rng, (width, C), "fp32")
    bias, bias64 = tensor(rng, (C,), "fp32")
    state, state64 = tensor(rng, (slots, width - 1, C), x_kind)
    ids = rng.permutation(slots)[:batch]
    if batch > 2:
        ids[1], ids[2] = -1, slots  # padding rows
    new = state if in_place else torch.full_like(state, 5.0)
    whole, y = guarded(batch * C, TYPES[y_kind])
    isam.conv1d_step(batch, C, width, slots, x, w, bias, True, torch.from_numpy(ids).int().cuda(), state, new, y)
    isam.sync()
    left = state64.copy() if in_place else np.full_like(state64, 5.0)
    want, size = np.zeros((batch, C)), np.zeros((batch, C))
    for i, slot in enumerate(ids):
        if 0 <= slot < slots:
            v, last, s = ref.conv(x64[None, i: i + 1], w64, bias64, True, state64[slot: slot + 1], np.ones(1))
            want[i], size[i], left[slot] = v[0, 0], s[0, 0], last[0]
    assert close(y.view(batch, C), want, ref.conv_bound(want, size, width, True, y_kind))
    assert close(new, left, 0.0)
    assert intact(whole, batch * C)


def test_tokens_after_a_prompt_are_the_longer_prompt():
    T, more, batch, C, width = 21, 6, 3, 96, 4
    rng = np.random.default_rng(7)
    x, _ = tensor(rng, (T + more, batch, C), "bf16")
    w, _ = tensor(rng, (width, C), "fp32")
    bias, _ = tensor(rng, (C,), "fp32")
    y = torch.empty(T + more, batch, C, device="cuda")
    isam.conv1d_forward(T + more, batch, C, width, x, w, bias, True, None, None, y)
    first, state = torch.empty(T, batch, C, device="cuda"), torch.empty(batch, width - 1, C, dtype=torch.bfloat16, device="cuda")
    isam.conv1d_forward(T, batch, C, width, x[:T], w, bias, True, None, None, first, state)
    got = [first]
    for t in range(T, T + more):
        one = torch.empty(batch, C, device="cuda")
        isam.conv1d_step(batch, C, width, batch, x[t], w, bias, True, None, state, state, one)
        got.append(one[None])
    assert torch.equal(torch.cat(got), y)


def test_long_and_many():
    """More runs of steps than a grid's second axis holds; many sequences."""
    rng = np.random.default_rng(8)
    for T, batch, C in ((1_200_003, 1, 4), (3, 30_000, 5)):
        x, _ = tensor(rng, (T, batch, C), "bf16")
        w, _ = tensor(rng, (2, C), "fp32")
        y = torch.empty(T, batch, C, device="cuda")
        isam.conv1d_forward(T, batch, C, 2, x, w, None, False, None, None, y)
        xf = x.float()
        before = torch.cat([torch.zeros_like(xf[:1]), xf[:-1]])
        want = before.double() * w[0].double() + xf.double() * w[1].double()
        size = before.double().abs() * w[0].abs() + xf.double().abs() * w[1].abs()
        assert bool(((y.double() - want).abs() <= 3 * ref.U * size + 1e-38).all())
