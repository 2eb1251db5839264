"""Beam search's selection and the reordering of states, against the
definition in 64 bits."""
import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_1810_09958_gb300 import isam
from test_norm_gpu import TYPES

pytestmark = pytest.mark.gpu


def run(logits, scores, count, eos=-1, finished=None, workspace=None):
    batch, beams, V = logits.shape
    out = (torch.full((batch, count), 5.0, device="cuda"), torch.full((batch, count), 7, dtype=torch.int32, device="cuda"),
           torch.full((batch, count), 7, dtype=torch.int32, device="cuda"), torch.full((batch, count), 7, dtype=torch.uint8, device="cuda"))
    isam.beam_select(batch, beams, V, count, logits, scores, eos, finished, *out, workspace)
    isam.sync()
    return [t.cpu().numpy() for t in out]


def check(logits, scores, count, eos=-1, finished=None):
    """Same choices as the 64-bit form wherever it sets neighbours apart by more than 32-bit sums can move them."""
    batch, beams, V = logits.shape
    got = run(logits, scores, count, eos, finished)
    l, s = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    ended = None if finished is None else finished.cpu().numpy()
    # The sum of exponentials: V / 256 + 64 additions, exp to 2^-21; its logarithm is off by as much.
    tol = (V / 256 + 64) * ref.U + 2.0 ** -21
    for b in range(batch):
        want = ref.select(l[b], s[b], eos, None if ended is None else ended[b], count + 1)
        for i in range(count):
            score, parent, token, end = want[i]
            if score == -np.inf:
                assert (got[0][b, i], got[1][b, i], got[2][b, i], got[3][b, i]) == (-np.inf, 0, 0, 0)
                continue
            assert abs(got[0][b, i] - score) <= tol + ref.U * abs(score)
            close_by = [w for w in want if abs(w[0] - score) <= 2 * tol and w[1] != parent]
            mine = (got[1][b, i], got[2][b, i], bool(got[3][b, i]))
            assert mine == (parent, token, end) or (close_by and mine in [w[1:] for w in close_by])


def logits_of(rng, shape, kind, scale=2.5):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(TYPES[kind]).cuda()


def scores_of(rng, shape):
    return torch.from_numpy(-np.sort(rng.uniform(0, 4, shape)).astype(np.float32)).cuda()


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("batch,beams,V,count", [
    (1, 1, 1, 1), (1, 1, 5, 8), (2, 3, 7, 3), (1, 4, 100, 8), (3, 2, 257, 4), (2, 5, 1000, 10), (1, 8, 4096, 16),
    (2, 4, 4097, 64), (1, 64, 513, 64), (4, 4, 32001, 4), (1, 3, 128003, 33), (40, 7, 3000, 7), (2, 16, 20000, 32),
    (300, 2, 50, 2)])
def test_select(batch, beams, V, count, kind):
    rng = np.random.default_rng(V + count)
    check(logits_of(rng, (batch, beams, V), kind), scores_of(rng, (batch, beams)), count)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [6, 1021, 40000])
def test_masks_ends_and_dead_beams(V, kind):
    rng = np.random.default_rng(V)
    batch, beams, count = 8, 5, 10
    l = logits_of(rng, (batch, beams, V), kind)
    l[0, :, ::3] = -float("inf")
    l[1, :, 1:] = -float("inf")        # one token left
    l[2] = -float("inf")               # nothing left
    l[3, 1] = -float("inf")
    l[3, 2, V // 2] = float("inf")     # no softmax
    l[4, :, ::2] = float("nan")
    l[4, 3] = float("nan")
    s = scores_of(rng, (batch, beams))
    s[5, 1], s[5, 2], s[5, 3] = -float("inf"), float("nan"), float("inf")
    finished = torch.from_numpy(rng.random((batch, beams)) < 0.3).cuda()
    finished[6] = True                 # all have ended: beams continuations, then nothing
    finished[2:6] = False
    finished[5, 4] = True
    check(l, s, count, 3, finished)
    check(l, s, count, 3, finished.to(torch.uint8) * 200)
    check(l, s, count, -1, None)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [37, 5003, 70001])
def test_masks_of_the_lowest_value(V, kind):
    """Tokens masked with the type's lowest value, rows that hold nothing else, rows of very large logits."""
    rng = np.random.default_rng(V)
    low = torch.finfo(TYPES[kind]).min
    l = logits_of(rng, (4, 3, V), kind)
    l[0, :, 1::2] = low
    l[1, 0] = low                       # uniform
    l[1, 1] = low
    l[1, 1, V // 3] = low / 2           # one token stands out
    l[2] = l[2] * 1e32                  # differences of 1e32: one token takes all
    l[3, :, ::5] = -1e35
    s = scores_of(rng, (4, 3))
    s[2] *= 1e33                        # (the sums of such rows are as large)
    check(l[:2], s[:2], 6)
    check(l[3:], s[3:], 6)
    got = run(l[2:3], s[2:3], 3)
    best = l[2].double().max(1)
    for k in range(3):                  # each beam's own best token costs nothing, and all others 1e30 or more
        at = [i for i in range(3) if got[1][0, i] == k]
        assert all(got[0][0, i] <= s[2, k].item() for i in at)
    assert got[2][0, 0] == best.indices[got[1][0, 0]].item()


def test_ties_go_to_the_lower_beam_and_token():
    V, beams = 5000, 4
    l = torch.zeros(1, beams, V, device="cuda")
    s = torch.zeros(1, beams, device="cuda")
    got = run(l, s, 16)
    assert (got[1] == 0).all() and (got[2][0] == np.arange(16)).all()
    l[0, 0, 100:] = -1.0    # beam 0's own best come first, then its rest loses to the others' equals
    l[0, 0, :100] = -0.0    # minus zero is zero
    l[0, 0, 7] = 0.0
    got = run(l[:, :1], s[:, :1], 16)
    assert (got[2][0] == np.arange(16)).all()
    same = torch.randn(V, device="cuda").sort(descending=True).values.repeat(1, beams, 1)
    got = run(same, s, 12)
    assert (got[1][0] == [0, 1, 2, 3] * 3).all() and (got[2][0] == np.repeat(np.arange(3), 4)).all()


@pytest.mark.parametrize("V", [30000, 200001])
@pytest.mark.parametrize("up", [False, True])
def test_sorted_rows(V, up):
    """Rows in order, the worst for a running threshold."""
    l = torch.linspace(-30, 30, V, device="cuda") * (1.0 if up else -1.0)
    l = torch.stack([l, l * 0.5])[None]
    check(l, torch.tensor([[0.0, -1.0]], device="cuda"), 32)


def test_in_place_and_replayed():
    rng = np.random.default_rng(3)
    batch, beams, V = 3, 4, 9000
    l = logits_of(rng, (batch, beams, V), "fp32")
    s, f = scores_of(rng, (batch, beams)), torch.zeros(batch, beams, dtype=torch.bool, device="cuda")
    f[1, 2] = True
    want = run(l, s.clone(), beams, 9, f.clone())
    parents, tokens = (torch.empty(batch, beams, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.empty(isam.beam_select_workspace(batch, beams, V, beams), dtype=torch.uint8, device="cuda")
    s2, f2 = s.clone(), f.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        isam.beam_select(batch, beams, V, beams, l, s2, 9, f2, s2, parents, tokens, f2, ws)
    graph.replay()
    torch.cuda.synchronize()
    for got, w in zip((s2, parents, tokens, f2), want):
        assert (got.cpu().numpy() == w).all()
    first = s2.clone()
    graph.replay()  # the next step from this one's scores
    torch.cuda.synchronize()
    again = run(l, first, beams, 9, torch.from_numpy(want[3] != 0).cuda())
    for got, w in zip((s2, parents, tokens, f2), again):
        assert (got.cpu().numpy() == w).all()


@pytest.mark.parametrize("dtype,row", [(torch.float32, 64), (torch.float32, 33), (torch.bfloat16, 33), (torch.uint8, 7),
                                       (torch.float32, 5000), (torch.bfloat16, 1)])
@pytest.mark.parametrize("layers,batch,beams", [(1, 1, 1), (3, 2, 4), (2, 5, 16), (1, 2, 64)])
@pytest.mark.parametrize("ids,in_place", [(True, False), (True, True), (False, True)])
def test_reorder(layers, batch, beams, dtype, row, ids, in_place):
    rng = np.random.default_rng(row + beams)
    n = batch * beams
    slots = n + 3
    state = torch.from_numpy(rng.integers(0, 120, (layers, slots, row))).to(dtype).cuda()
    slot = rng.permutation(slots)[:n].reshape(batch, beams) if ids else np.arange(n).reshape(batch, beams)
    parents = rng.integers(0, beams, (batch, beams))
    if beams > 2:
        parents[0, 1], parents[-1, 2] = -1, beams  # left as they are
        if ids:
            slot[0, 0], slot[-1, 1] = -1, slots + 5  # padding, as itself and as a parent
            parents[0, 2] = 0
    new = state if in_place else torch.full_like(state, 3)
    old = state.cpu().clone()
    want = old.clone() if in_place else new.cpu().clone()
    for b in range(batch):
        for k in range(beams):
            p = parents[b, k]
            if 0 <= p < beams and 0 <= slot[b, k] < slots and 0 <= slot[b, p] < slots:
                want[:, slot[b, k]] = old[:, slot[b, p]]
    isam.beam_reorder(layers, batch, beams, slots, torch.from_numpy(parents).int().cuda(),
                      torch.from_numpy(slot).int().cuda() if ids else None, state, new)
    isam.sync()
    assert torch.equal(new.cpu(), want)


def test_reorder_past_32_bits():
    """A cache above 4 GB."""
    layers, beams, row = 3, 4, 500_000_000
    if torch.cuda.mem_get_info()[0] < 30e9:
        pytest.skip("needs 30 GB")
    state = torch.zeros(layers, beams, row, dtype=torch.uint8, device="cuda")
    state += torch.arange(layers * beams, dtype=torch.uint8, device="cuda").view(layers, beams, 1)
    isam.beam_reorder(layers, 1, beams, beams, torch.tensor([[3, 3, 0, 1]], dtype=torch.int32, device="cuda"), None, state, state)
    isam.sync()
    for layer in range(layers):
        for k, p in enumerate((3, 3, 0, 1)):
            assert bool((state[layer, k] == layer * beams + p).all())
