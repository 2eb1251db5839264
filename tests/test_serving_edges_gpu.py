"""Calls of the norm, the convolution, the scan and beam search that users may make
besides the plain ones: tensors off 16-byte boundaries, several threads on streams
of their own, captured graphs that share a workspace, calls that follow each other on one stream."""
import threading

import numpy as np
import pytest
import torch

from paper_1810_09958_gb300 import isam

pytestmark = pytest.mark.gpu


def shifted(t, by):
    """A contiguous copy of t that begins `by` elements behind a boundary."""
    whole = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
    part = whole[by:].view(t.shape)
    part.copy_(t)
    return part


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("by", [1, 2, 4])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_norm_off_boundaries(by, kind):
    """Other places give other loads and orders of sums, no other results than rounding's: 96 half steps and the type's."""
    T, D = 9, 256
    x, res, w, dy = normal(1, T, D).to(kind), normal(2, T, D).to(kind), normal(3, D), normal(4, T, D).to(kind)
    tol = 96 * 2.0 ** -24 + 2 * (2.0 ** -8 if kind == torch.bfloat16 else 0)

    def call(f):
        y, r, dx, dw = f(torch.empty_like(x)), f(torch.empty_like(x)), f(torch.empty_like(x)), f(torch.empty_like(w))
        isam.rms_norm_forward(T, D, f(x), f(res), r, f(w), 1e-5, y)
        isam.rms_norm_backward(T, D, f(x), f(w), 1e-5, f(dy), f(res), dx, dw)
        return y, r, dx, dw

    for a, b in zip(call(lambda t: t), call(lambda t: shifted(t, by))):
        assert float((a.double() - b.double()).abs().max()) <= tol * float(a.double().abs().max())
    q, s = torch.empty(T, D, dtype=torch.uint8, device="cuda"), torch.empty(2, T, 4, dtype=torch.uint8, device="cuda")
    q2, s2 = shifted(q, 3), shifted(s, 4)
    isam.rms_norm_forward(T, D, x, res, None, w, 1e-5, None, q, s)
    isam.rms_norm_forward(T, D, x, res, None, w, 1e-5, None, q2, s2)
    assert float((s != s2).float().mean()) <= 0.02 and float((q != q2).float().mean()) <= 0.02  # (sums' orders differ)


@pytest.mark.parametrize("by", [1, 2])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_convolution_and_scan_off_boundaries(by, kind):
    T, batch, C, N, W = 75, 2, 96, 16, 4
    x, dt, z, bc = (normal(i, T, batch, n).to(kind) for i, n in enumerate((C, C, C, 2 * N)))
    w, bias, A, D, state = normal(5, W, C), normal(6, C), -normal(7, C, N).abs(), normal(8, C), normal(9, batch, W - 1, C).to(kind)
    h0 = normal(10, batch, C, N)

    def call(f):
        u, new, y, last = (f(torch.empty(*s, dtype=k, device="cuda")) for s, k in (
            ((T, batch, C), kind), ((batch, W - 1, C), kind), ((T, batch, C), kind), ((batch, C, N), torch.float32)))
        isam.conv1d_forward(T, batch, C, W, f(x), f(w), f(bias), True, f(state), None, u, new)
        b = f(bc)
        isam.ssm_forward(T, batch, C, N, u, f(dt), f(bias), f(A), b[..., :N], b[..., N:], f(D), f(z), f(h0), None, y, last)
        cache, out = f(h0.clone()), f(torch.empty(batch, C, dtype=kind, device="cuda"))
        one = f(bc[0].contiguous())
        isam.ssm_step(batch, C, N, batch, f(u[0].contiguous()), f(dt[0].contiguous()), f(bias), f(A), one[:, :N], one[:, N:],
                      f(D), f(z[0].contiguous()), None, cache, cache, out)
        return u, new, y, last, cache, out

    # fp32: sums in other orders; bf16: a rounding may fall to the other side.
    tol = 2.0 ** -18 if kind == torch.float32 else 2.0 ** -7
    for a, b in zip(call(lambda t: t), call(lambda t: shifted(t, by))):
        assert float((a.double() - b.double()).abs().max()) <= tol * float(a.double().abs().max())


@pytest.mark.parametrize("by", [1, 2, 3, 5])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_selection_off_boundaries(by, kind):
    batch, beams, V, count = 2, 3, 9001, 6
    logits, scores = normal(1, batch, beams, V).to(kind), normal(2, batch, beams)

    def call(l):
        out = [torch.empty(batch, count, dtype=k, device="cuda") for k in (torch.float32, torch.int32, torch.int32)]
        isam.beam_select(batch, beams, V, count, l, scores, -1, None, *out)
        return out

    a, b = call(logits), call(shifted(logits, by))
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    assert float((a[0] - b[0]).abs().max()) <= 2e-5  # (sums of 9001 exponentials in another order)


def test_threads_on_streams_of_their_own():
    T, batch, C, N, V = 130, 2, 64, 16, 4000
    u, dt, bc, A = normal(1, T, batch, C), normal(2, T, batch, C), normal(3, T, batch, 2 * N), -normal(4, C, N).abs()
    logits, scores, r, w = normal(5, 4, 4, V), normal(6, 4, 4), normal(7, 300, 320), normal(8, 320)

    def work():
        y, last = torch.empty(T, batch, C, device="cuda"), torch.empty(batch, C, N, device="cuda")
        isam.ssm_forward(T, batch, C, N, u, dt, None, A, bc[..., :N], bc[..., N:], None, None, None, None, y, last)
        best = [torch.empty(4, 8, dtype=k, device="cuda") for k in (torch.float32, torch.int32, torch.int32)]
        isam.beam_select(4, 4, V, 8, logits, scores, -1, None, *best)
        dx, dw = torch.empty_like(r), torch.empty_like(w)
        isam.rms_norm_backward(300, 320, r, w, 1e-5, r, None, dx, dw)
        return [y, last, *best, dx, dw]

    want = work()
    torch.cuda.synchronize()
    got, failed = {}, []

    def run(i):
        try:
            torch.cuda.set_device(0)
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[i] = work()
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for i in range(3):
        for a, b in zip(got[i], want):
            assert torch.equal(a, b)


def test_graphs_that_share_a_workspace():
    """Two captured calls with one workspace, replayed in turn on one stream."""
    batch, beams, V, T, D = 3, 4, 20000, 200, 520
    ws = torch.empty(max(isam.beam_select_workspace(batch, beams, V, beams), isam.rms_norm_backward_workspace(T, D)),
                     dtype=torch.uint8, device="cuda")
    logits, scores, r, w, dy = normal(1, batch, beams, V), normal(2, batch, beams), normal(3, T, D), normal(4, D), normal(5, T, D)
    out = [[torch.empty(batch, beams, dtype=k, device="cuda") for k in (torch.float32, torch.int32, torch.int32)] for _ in range(2)]
    dx, dw = [torch.empty_like(r) for _ in range(2)], [torch.empty_like(w) for _ in range(2)]

    def calls(i, workspace):
        isam.beam_select(batch, beams, V, beams, logits, scores, -1, None, *out[i], None, workspace)
        isam.rms_norm_backward(T, D, r, w, 1e-5, dy, None, dx[i], dw[i], workspace)

    calls(0, None)
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        isam.beam_select(batch, beams, V, beams, logits, scores, -1, None, *out[1], None, ws)
    with torch.cuda.graph(second):
        isam.rms_norm_backward(T, D, r, w, 1e-5, dy, None, dx[1], dw[1], ws)
    for _ in range(5):
        first.replay()
        second.replay()
    torch.cuda.synchronize()
    for a, b in zip(out[0] + [dx[0], dw[0]], out[1] + [dx[1], dw[1]]):
        assert torch.equal(a, b)
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="are needed"):
        calls(0, small)


def test_results_feed_the_next_call_at_once():
    """Kernels start before their predecessors have ended and wait for them: a chain without a pause, many times."""
    T, D = 64, 1024
    x, w = normal(1, T, D), torch.ones(D, device="cuda")
    a, b = torch.empty(T, D, device="cuda"), torch.empty(T, D, device="cuda")
    for _ in range(200):
        isam.rms_norm_forward(T, D, x, None, None, w, 0.0, a)
        isam.rms_norm_forward(T, D, a, a, b, w, 0.0, x)
    isam.sync()
    want = normal(1, T, D).double()
    want = want / want.square().mean(1, keepdim=True).sqrt()
    assert float((x.double() - want).abs().max()) <= 400 * 48 * 2.0 ** -24 * float(want.abs().max())


def test_rows_of_wider_tensors_are_checked():
    x = normal(1, 6, 4, 80).bfloat16()
    w, y = normal(2, 4, 40), torch.empty(6, 4, 40, device="cuda")
    isam.conv1d_forward(6, 4, 40, 4, x[..., 40:], w, None, False, None, None, y)
    for bad in (x.transpose(0, 1)[..., :40], x[..., ::2], x[:, :, :40].transpose(1, 2)):
        with pytest.raises(ValueError, match="x "):
            isam.conv1d_forward(*((6, 4) if bad.shape[0] == 6 else (4, 6)), 40, 4, bad, w, None, False, None, None, y)
    with pytest.raises(ValueError, match="equally far apart"):
        n = normal(3, 6, 4, 16).bfloat16()
        isam.ssm_forward(6, 4, 40, 16, y, normal(4, 6, 4, 40).bfloat16(), None, normal(5, 40, 16), n, x[..., :16], None, None, None,
                         None, y)


def room(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 1e9:
        pytest.skip(f"needs {gigabytes} GB")


def test_selection_past_32_bits():
    """More than 2^31 logits: the last sequence's choice is that of a call of its own."""
    room(12)
    batch, beams, V, count = 275, 4, 2_000_003, 5
    logits = torch.empty(batch, beams, V, dtype=torch.bfloat16, device="cuda")
    logits.zero_()
    logits[-1] = normal(1, beams, V).bfloat16()
    scores = normal(2, batch, beams)

    def call(n, l, s):
        out = [torch.empty(n, count, dtype=k, device="cuda") for k in (torch.float32, torch.int32, torch.int32)]
        isam.beam_select(n, beams, V, count, l, s, -1, None, *out)
        return out

    many, one = call(batch, logits, scores), call(1, logits[-1:].clone(), scores[-1:].clone())
    assert torch.equal(many[1][-1:], one[1]) and torch.equal(many[2][-1:], one[2])
    assert float((many[0][-1:] - one[0]).abs().max()) <= 1e-4
    assert torch.equal(many[2][0], torch.arange(count, dtype=torch.int32, device="cuda"))


def test_sequences_past_32_bits():
    """More than 2^31 values: the last steps are those of a call that goes on from the state before them."""
    room(40)
    T, C, N, W, tail = 1_100_000, 2048, 4, 4, 300
    x = torch.empty(T, 1, C, dtype=torch.bfloat16, device="cuda").normal_()
    w, bias = normal(1, W, C), normal(2, C)
    u = torch.empty_like(x)
    isam.conv1d_forward(T, 1, C, W, x, w, bias, True, None, None, u)
    few = torch.empty(tail, 1, C, dtype=torch.bfloat16, device="cuda")
    isam.conv1d_forward(tail, 1, C, W, x[T - tail:], w, bias, True, x[T - tail - W + 1: T - tail].view(1, W - 1, C), None, few)
    assert torch.equal(u[T - tail:], few)
    bc, A, y, last = normal(3, T, 1, 2 * N).bfloat16(), -normal(4, C, N).abs() - 0.1, torch.empty_like(x), torch.empty(1, C, N, device="cuda")
    B, Cm = bc[..., :N], bc[..., N:]
    isam.ssm_forward(T, 1, C, N, u, x, None, A, B, Cm, bias, None, None, None, y, last)
    before, end = torch.empty(1, C, N, device="cuda"), torch.empty(1, C, N, device="cuda")
    isam.ssm_forward(T - tail, 1, C, N, u[:T - tail], x[:T - tail], None, A, B[:T - tail], Cm[:T - tail], bias, None, None, None,
                     y[:T - tail], before)
    isam.ssm_forward(tail, 1, C, N, u[T - tail:], x[T - tail:], None, A, B[T - tail:], Cm[T - tail:], bias, None, before, None, few, end)
    # Other cuts of time: starts differ by roundings of states that decay; y by a rounding to bf16 either way.
    assert float((end - last).abs().max()) <= 2.0 ** -18 * float(last.abs().max())
    assert float((few.float() - y[T - tail:].float()).abs().max()) <= 2.0 ** -7 * float(few.abs().max())


def test_a_cache_past_32_bits():
    """Slots above 2^31 states."""
    room(30)
    C, N, slots = 4096, 16, 40_000
    state = torch.empty(slots, C, N, device="cuda")
    ids = torch.tensor([slots - 1, 3, -1, slots - 2], dtype=torch.int32, device="cuda")
    state[ids[ids >= 0].long()] = normal(1, 3, C, N)
    small = torch.stack([state[slots - 1], state[3], state[slots - 2]])
    u, dt, bc, A = normal(2, 4, C), normal(3, 4, C), normal(4, 4, 2 * N), -normal(5, C, N).abs()
    y, y2 = torch.empty(4, C, device="cuda"), torch.empty(4, C, device="cuda")
    isam.ssm_step(4, C, N, slots, u, dt, None, A, bc[:, :N], bc[:, N:], None, None, ids, state, state, y)
    isam.ssm_step(4, C, N, 3, u, dt, None, A, bc[:, :N], bc[:, N:], None, None,
                  torch.tensor([0, 1, -1, 2], dtype=torch.int32, device="cuda"), small, small, y2)
    assert torch.equal(y, y2) and torch.equal(state[slots - 1], small[0]) and torch.equal(state[slots - 2], small[2])
    del state
