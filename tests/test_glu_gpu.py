"""The gated feed-forward product and its backward pass on the GPU against the
definition in 64 bits.

Tolerances.  The sums over D (at most 2048 here) are fp32 on the tensor cores:
each of D additions loses at most 2^-23, all in one direction 2^-12 of the
largest value.  Results are rounded to bf16 (8 significant bits: at most 2^-8
of themselves).  In the backward pass d = [dg | du] is rounded to bf16 before
the second products: each term is off by at most 2^-8 of itself,
independently, so a sum is off by about 2^-8 / sqrt(3) * sqrt(sum of squared
terms); six times that is allowed."""
import numpy as np
import pytest

import lm_ref
from gpu_util import CANARY
from paper_1810_09958_gb300 import isam

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "relu", "sigmoid"]
SUM = 2.0 ** -12
BF16 = 2.0 ** -8
PAD = 64


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import torch
    from paper_1810_09958_gb300 import build
    build.build()
    isam.load()
    torch.cuda.set_device(0)
    yield
    isam.sync()


def guarded(shape):
    import torch
    n = int(np.prod(shape))
    buf = torch.full((n + 2 * PAD,), CANARY, dtype=torch.bfloat16, device="cuda")
    buf[PAD:PAD + n] = float("nan")
    return buf, buf[PAD:PAD + n]


def intact(buf, n):
    c = buf.new_tensor(CANARY)
    return bool((buf[:PAD] == c).all()) and bool((buf[PAD + n:] == c).all())


def operands(T, D, F, seed):
    import torch
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((T, D))).bfloat16()
    W = torch.from_numpy(rng.standard_normal((2 * F, D)) / np.sqrt(D)).bfloat16()
    dh = torch.from_numpy(rng.standard_normal((T, F))).bfloat16()
    return x, W, dh


def f64(t):
    return t.double().cpu().numpy()


def check_forward(T, D, F, act, seed=1):
    x, W, _ = operands(T, D, F, seed)
    buf, h = guarded((T, F))
    isam.glu_forward(T, D, F, act, x.cuda(), W.cuda(), h)
    isam.sync()
    ref = lm_ref.glu(f64(x), f64(W), act)
    got = f64(h).reshape(T, F)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= BF16 * np.abs(ref) + SUM * np.abs(ref).max()).all()
    assert intact(buf, T * F)


def check_backward(T, D, F, act, seed=2, want=("dx", "dW")):
    import torch
    x, W, dh = operands(T, D, F, seed)
    bx, dx = guarded((T, D))
    bw, dW = guarded((2 * F, D))
    ws = torch.full((isam.glu_backward_workspace(T, D, F) + 256,), 0xC5, dtype=torch.uint8, device="cuda")
    need = ws.numel() - 256
    isam.glu_backward(T, D, F, act, x.cuda(), W.cuda(), dh.cuda(), dx if "dx" in want else None,
                      dW if "dW" in want else None, workspace=ws[:need])
    isam.sync()
    rx, rw, d = lm_ref.glu_backward(f64(x), f64(W), f64(dh), act)
    noise = 6 * 2.0 ** -8 / np.sqrt(3)
    for name, got, ref, sq in (("dx", dx, rx, (d ** 2) @ (f64(W) ** 2)), ("dW", dW, rw, (d ** 2).T @ (f64(x) ** 2))):
        got = f64(got).reshape(ref.shape)
        if name not in want:
            assert np.isnan(got).all()
            continue
        assert np.isfinite(got).all()
        tol = BF16 * np.abs(ref) + noise * np.sqrt(sq) + SUM * np.abs(ref).max()
        assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / tol).max())
    assert intact(bx, T * D) and intact(bw, 2 * F * D)
    assert bool((ws[need:] == 0xC5).all())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,D,F", [(1, 8, 1), (3, 64, 17), (20, 200, 72), (130, 136, 130)])
def test_forward_activations(T, D, F, act):
    check_forward(T, D, F, act)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300])
def test_forward_tokens(T):
    check_forward(T, 328, 200, "silu", seed=T)


@pytest.mark.parametrize("F", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 333, 1000])
def test_forward_features(F):
    check_forward(5, 136, F, "gelu", seed=F)
    check_forward(150, 72, F, "relu", seed=F)


@pytest.mark.parametrize("D", [8, 16, 56, 64, 72, 120, 128, 136, 512, 1024, 1032, 2048])
def test_forward_depths(D):
    check_forward(4, D, 96, "silu", seed=D)
    check_forward(140, D, 96, "sigmoid", seed=D)


@pytest.mark.parametrize("T,D,F", [(1, 2048, 1024), (512, 512, 768), (1024, 1024, 1000), (2500, 256, 520)])
def test_forward_ordinary(T, D, F):
    check_forward(T, D, F, "silu")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,D,F", [(1, 8, 8), (5, 72, 16), (70, 200, 136), (130, 136, 264)])
def test_backward_activations(T, D, F, act):
    check_backward(T, D, F, act)


@pytest.mark.parametrize("T", [1, 2, 8, 17, 32, 33, 64, 65, 127, 128, 129, 255, 257, 700])
def test_backward_tokens(T):
    check_backward(T, 264, 152, "silu", seed=T)


@pytest.mark.parametrize("T,D,F", [(40, 8, 2000), (40, 2000, 8), (2000, 8, 8), (512, 512, 768), (300, 1024, 1000),
                                   (1100, 648, 520)])
def test_backward_shapes(T, D, F):
    check_backward(T, D, F, "gelu")


@pytest.mark.parametrize("T,D,F", [(300, 4360, 1400), (270, 2056, 520), (129, 264, 4096), (128, 520, 2048),
                                   (2300, 1032, 264), (90, 8, 4096), (1300, 520, 1536 + 8), (2400, 2056, 2048)])
def test_backward_split_sums(T, D, F):
    """Shapes whose products leave a round of tiles part empty, so that tiles are
    summed in parts: whole rounds before them, none before them, edges in them."""
    check_backward(T, D, F, "silu", seed=T + D)


@pytest.mark.parametrize("T", [3, 4, 5, 6, 15, 16, 18, 31, 32])
@pytest.mark.parametrize("D,F", [(8, 8), (504, 24), (520, 1000), (1032, 136), (2048, 64)])
def test_backward_few_tokens(T, D, F):
    check_backward(T, D, F, "silu", seed=T + F)


@pytest.mark.parametrize("want", [("dx",), ("dW",), ()])
def test_backward_of_one_operand(want):
    check_backward(70, 72, 40, "silu", want=want)


def test_integer_data():
    """Small integers: every sum is exact, so relu's result is its bf16 rounding."""
    import torch
    T, D, F = 200, 136, 72
    rng = np.random.default_rng(8)
    x = torch.from_numpy(rng.integers(-2, 3, (T, D)).astype(np.float32)).bfloat16()
    W = torch.from_numpy(rng.integers(-1, 2, (2 * F, D)).astype(np.float32)).bfloat16()
    ref = torch.from_numpy(lm_ref.glu(f64(x), f64(W), "relu")).to(torch.float32).bfloat16()
    for rows in (1, 8, 40, 200):
        h = torch.empty(rows, F, dtype=torch.bfloat16, device="cuda")
        isam.glu_forward(rows, D, F, "relu", x[:rows].cuda(), W.cuda(), h)
        isam.sync()
        assert torch.equal(h.cpu(), ref[:rows])


def test_gradient_against_differences():
    """Directional derivatives of the 64-bit form by central differences; the
    gradient's own tolerance is that of its bf16 rounding and of d's, 2^-8 of
    each of the terms, which add up independently."""
    import torch
    T, D, F = 24, 40, 32
    rng = np.random.default_rng(5)
    for act in ("silu", "gelu", "sigmoid"):
        x, W, dh = operands(T, D, F, seed=6)
        dx = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
        dW = torch.empty(2 * F, D, dtype=torch.bfloat16, device="cuda")
        isam.glu_backward(T, D, F, act, x.cuda(), W.cuda(), dh.cuda(), dx, dW)
        isam.sync()
        for _ in range(4):
            v, w = rng.standard_normal((T, D)), rng.standard_normal((2 * F, D))
            eps = 1e-4
            num = ((lm_ref.glu(f64(x) + eps * v, f64(W) + eps * w, act) -
                    lm_ref.glu(f64(x) - eps * v, f64(W) - eps * w, act)) * f64(dh)).sum() / (2 * eps)
            got = (f64(dx) * v).sum() + (f64(dW) * w).sum()
            size = np.sqrt(((f64(dx) * v) ** 2).sum() + ((f64(dW) * w) ** 2).sum())
            assert abs(got - num) <= 6 * 2.0 ** -8 * size + 1e-6 * abs(num)


def test_infinities_and_nan_stay_in_their_row():
    import torch
    D, F = 136, 72
    for T in (5, 150):
        x, W, _ = operands(T, D, F, seed=7)
        h0, h1 = (torch.empty(T, F, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        isam.glu_forward(T, D, F, "silu", x.cuda(), W.cuda(), h0)
        x[3, 9] = float("nan")
        isam.glu_forward(T, D, F, "silu", x.cuda(), W.cuda(), h1)
        isam.sync()
        rest = [t for t in range(T) if t != 3]
        assert torch.equal(h0[rest], h1[rest]) and torch.isnan(h1[3]).all()


def test_same_bits_on_another_stream():
    import torch
    for T, D, F in ((3, 1024, 520), (100, 1024, 520), (600, 520, 776)):
        x, W, dh = (t.cuda() for t in operands(T, D, F, seed=9))
        outs = []
        for st in (torch.cuda.current_stream(), torch.cuda.Stream()):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                h, dx, dW = torch.empty_like(dh), torch.empty_like(x), torch.empty_like(W)
                isam.glu_forward(T, D, F, "silu", x, W, h)
                isam.glu_backward(T, D, F, "silu", x, W, dh, dx, dW)
                isam.sync()
            outs.append((h, dx, dW))
        for a, b in zip(*outs):
            assert torch.equal(a, b)


def test_captured_in_a_graph():
    import torch
    T, D, F = 64, 264, 136
    x, W, dh = (t.cuda() for t in operands(T, D, F, seed=10))
    h, dx, dW = torch.empty_like(dh), torch.empty_like(x), torch.empty_like(W)
    ws = torch.empty(isam.glu_backward_workspace(T, D, F), dtype=torch.uint8, device="cuda")

    def both():
        isam.glu_forward(T, D, F, "silu", x, W, h)
        isam.glu_backward(T, D, F, "silu", x, W, dh, dx, dW, workspace=ws)

    both()
    isam.sync()
    want = [t.clone() for t in (h, dx, dW)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for t in (h, dx, dW):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, (h, dx, dW)):
        assert torch.equal(a, b)


def test_backward_takes_its_workspace_from_the_allocator():
    """Without a workspace argument: the same bits, on another stream and in a
    captured graph too, and nothing left allocated."""
    import torch
    T, D, F = 300, 520, 264
    x, W, dh = (t.cuda() for t in operands(T, D, F, 5))
    want = torch.empty_like(x), torch.empty_like(W)
    ws = torch.empty(isam.glu_backward_workspace(T, D, F), dtype=torch.uint8, device="cuda")
    isam.glu_backward(T, D, F, "silu", x, W, dh, *want, workspace=ws)
    isam.sync()

    def same(got):
        return all(torch.equal(a, b) for a, b in zip(got, want))
    before = torch.cuda.memory_allocated()
    got = torch.zeros_like(x), torch.zeros_like(W)
    held = torch.cuda.memory_allocated() - before
    isam.glu_backward(T, D, F, "silu", x, W, dh, *got)
    assert torch.cuda.memory_allocated() - before == held
    isam.sync()
    assert same(got)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in got:
            t.zero_()
        for _ in range(3):
            isam.glu_backward(T, D, F, "silu", x, W, dh, *got)
    side.synchronize()
    assert same(got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        isam.glu_backward(T, D, F, "silu", x, W, dh, *got)
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert same(got)


def test_two_threads_on_streams_of_their_own():
    """The backward pass with the allocator's workspace from two threads at once,
    each reusing that memory between its calls: the bits of one thread alone."""
    import threading
    import torch
    T, D, F = 300, 520, 264
    ops = [[t.cuda() for t in operands(T, D, F, seed)] for seed in (11, 12)]
    want = []
    for x, W, dh in ops:
        dx, dW = torch.empty_like(x), torch.empty_like(W)
        isam.glu_backward(T, D, F, "silu", x, W, dh, dx, dW)
        isam.sync()
        want.append((dx, dW))
    got, failed = [[], []], []

    def work(i):
        try:
            torch.cuda.set_device(0)
            x, W, dh = ops[i]
            size = isam.glu_backward_workspace(T, D, F)
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(50):
                    dx, dW = torch.empty_like(x), torch.empty_like(W)
                    isam.glu_backward(T, D, F, "silu", x, W, dh, dx, dW)
                    torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")  # takes what the call gave back
                    got[i].append((dx, dW))
                stream.synchronize()
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    torch.cuda.synchronize()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    isam.sync()
    assert not failed, failed
    for outs, ref in zip(got, want):
        assert len(outs) == 50
        assert all(torch.equal(a, b) for o in outs for a, b in zip(o, ref))


@pytest.mark.parametrize("T", [1, 20, 150])
def test_gelu_far_below_zero(T):
    """GELU's tail is a product of a and a probability of 0.3 down to 1e-19: it is
    held to its own size, not to the largest output.  One product makes each gate
    sum, and u = 1, so h = gelu(x0 w): one rounding to bf16 (2^-8) beside a few
    fp32 operations (the probability's argument, off by 2^-24 of itself, counts
    a^2 <= 82 times: 2^-16 with the rest).  The same for du = dh gelu(x0 w), read
    off dW's up rows: only the first token has a gradient, of 1, and x1 = 1.  dW's gate rows then are
    gelu'(w), the sum of two terms of opposite sign that below -1.5 are together
    at most 2.1 times as large as it."""
    import math
    import torch
    D, F = 16, 96
    x, W = torch.zeros(T, D), torch.zeros(2 * F, D)
    x[:, 0] = 1 + (torch.arange(T) % 8) / 128
    x[:, 1] = 1
    W[:F, 0] = -torch.linspace(0.5, 8.5, F)
    W[F:, 1] = 1
    x, W = x.bfloat16().cuda(), W.bfloat16().cuda()
    a = f64(x)[:, :1] * f64(W)[None, :F, 0]
    ref = np.vectorize(lambda v: 0.5 * v * math.erfc(-v / math.sqrt(2)))(a)
    tol = (2.0 ** -8 + 2.0 ** -16) * np.abs(ref)
    buf, h = guarded((T, F))
    isam.glu_forward(T, D, F, "gelu", x, W, h)
    dh = torch.zeros(T, F, dtype=torch.bfloat16, device="cuda")
    dh[0] = 1
    dx, dW = torch.empty_like(x), torch.empty_like(W)
    isam.glu_backward(T, D, F, "gelu", x, W, dh, dx, dW)
    isam.sync()
    got, dup, dgate = f64(h).reshape(T, F), f64(dW)[F:, 1], f64(dW)[:F, 0]
    assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / np.abs(ref)).max())
    assert (np.abs(dup - ref[0]) <= tol[0]).all(), float((np.abs(dup - ref[0]) / np.abs(ref[0])).max())
    a0 = a[0]
    slope = ref[0] / a0 + a0 * np.exp(-a0 * a0 / 2) / math.sqrt(2 * math.pi)
    low = a0 < -1.5
    assert (np.abs(dgate - slope) <= (2.0 ** -8 + 2.1 * 2.0 ** -16) * np.abs(slope))[low].all()
    assert intact(buf, T * F)


@pytest.mark.parametrize("T", [1, 4, 5])
def test_backward_of_very_deep_rows(T):
    """More columns of dW than a grid has rows of blocks (65535 of 1024): x and W
    are integers in a few columns and zero elsewhere, so every result is exact
    and small."""
    import torch
    D, F = 65536 * 1024 + 8, 8
    at = [0, 1, 1023, D // 2, D - 9, D - 8, D - 1]
    rng = np.random.default_rng(T)
    xs = rng.integers(-1, 2, (T, len(at))).astype(np.float64)
    ws = rng.integers(-1, 2, (2 * F, len(at))).astype(np.float64)
    x, W = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(2 * F, D, dtype=torch.bfloat16, device="cuda")
    x[:, at], W[:, at] = torch.from_numpy(xs).bfloat16().cuda(), torch.from_numpy(ws).bfloat16().cuda()
    dh = torch.from_numpy(rng.integers(-1, 2, (T, F)).astype(np.float64)).bfloat16().cuda()
    dx, dW = torch.full_like(x, float("nan")), torch.full_like(W, float("nan"))
    isam.glu_backward(T, D, F, "relu", x, W, dh, dx, dW)
    isam.sync()
    rx, rw, d = lm_ref.glu_backward(xs, ws, f64(dh), "relu")
    exact = lambda v: torch.from_numpy(v).float().bfloat16().double().numpy()
    assert np.abs(d).max() < 256
    assert np.array_equal(f64(dx[:, at]), exact(rx)) and np.array_equal(f64(dW[:, at]), exact(rw))
    dx[:, at], dW[:, at] = 0, 0
    assert not dx.any() and not dW.any()
