"""The gated linear recurrence (forward, backward, one token on a state cache)
on the GPU against its definition in 64 bits.

Tolerances.  A step's update gate is within 2^-21 of itself (an exponential
and a quotient of a few units in the last place), and a state forgets: with
the gates drawn here (sigmoid of N(2, 1.5) per step) errors older than 64
steps have decayed away, so fp32 results are held to 64 * 2^-21 of the largest
value.  A bf16 result adds its rounding, 2^-8 of itself."""
import numpy as np
import pytest

import lm_ref
from gpu_util import CANARY
from paper_1810_09958_gb300 import isam

pytestmark = pytest.mark.gpu
F32 = 64 * 2.0 ** -21
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


def guarded(shape, dtype):
    """An output between two runs of canaries, filled with NaN."""
    import torch
    n = int(np.prod(shape))
    buf = torch.full((n + 2 * PAD,), CANARY, dtype=dtype, device="cuda")
    buf[PAD:PAD + n] = float("nan")
    return buf, buf[PAD:PAD + n]


def intact(buf, n):
    c = buf.new_tensor(CANARY)
    return bool((buf[:PAD] == c).all()) and bool((buf[PAD + n:] == c).all())


def tdtype(name):
    import torch
    return torch.float32 if name == "f32" else torch.bfloat16


def close(got, ref, bits16):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert np.isfinite(got).all()
    tol = F32 * np.max(np.abs(ref), initial=0) + (BF16 * np.abs(ref) if bits16 else 0) + 1e-30
    assert (np.abs(got - ref) <= tol).all(), float(np.max(np.abs(got - ref) - tol))


def make(T, B, H, gt, ht, seed, lengths=None, shift=2.0, scale=1.5):
    import torch
    rng = np.random.default_rng(seed)
    g = rng.standard_normal((T, B, 2 * H))
    g[:, :, :H] = g[:, :, :H] * scale + shift
    g = torch.from_numpy(g).to(tdtype(gt))
    h0 = torch.from_numpy(rng.standard_normal((B, H)).astype(np.float32))
    n = np.full(B, T) if lengths is None else np.asarray(lengths)
    dh = torch.from_numpy(rng.standard_normal((T, B, H))).to(tdtype(ht))
    dl = torch.from_numpy(rng.standard_normal((B, H)).astype(np.float32))
    return g, h0, n, dh, dl


def f64(t):
    return t.double().numpy()


def check_both(T, B, H, gt, ht, seed, lengths=None, use_h0=True, use_last=True, poison=float("nan")):
    import torch
    g, h0, n, dh, dl = make(T, B, H, gt, ht, seed, lengths)
    nc = np.clip(n, 0, T)
    zeros = np.zeros((B, H))
    out, last = lm_ref.recurrence(f64(g), f64(h0) if use_h0 else zeros, nc)
    gd, dhd = g.cuda(), dh.cuda()
    pad = torch.from_numpy(np.arange(T)[:, None] >= nc[None, :]).cuda()
    gd[pad], dhd[pad] = poison, poison
    ld = None if lengths is None else torch.from_numpy(n.astype(np.int32)).cuda()
    h0d = h0.cuda() if use_h0 else None
    hb, h = guarded((T, B, H), tdtype(ht))
    lb, hl = guarded((B, H), torch.float32)
    isam.glr_forward(T, B, H, gd, h0d, ld, h, hl if use_last else None)
    isam.sync()
    close(h.float().cpu().numpy().reshape(T, B, H), out, ht == "bf16")
    assert not h.view(T, B, H)[pad].any()
    assert intact(hb, T * B * H) and intact(lb, B * H)
    if use_last:
        close(hl.cpu().numpy().reshape(B, H), last, False)
        untouched = nc == 0
        if use_h0 and untouched.any():
            assert np.array_equal(hl.cpu().numpy().reshape(B, H)[untouched], h0.numpy()[untouched])

    saved = h.clone()
    saved.view(T, B, H)[pad] = poison  # not read in padding
    dg_ref, dh0_ref = lm_ref.recurrence_backward(f64(g), f64(h0) if use_h0 else zeros, nc,
                                                 h.double().cpu().numpy().reshape(T, B, H), f64(dh),
                                                 f64(dl) if use_last else zeros)
    gb, dg = guarded((T, B, 2 * H), tdtype(gt))
    eb, dh0 = guarded((B, H), torch.float32)
    isam.glr_backward(T, B, H, gd, h0d, ld, saved, dhd, dl.cuda() if use_last else None, dg, dh0)
    isam.sync()
    close(dg.float().cpu().numpy().reshape(T, B, 2 * H), dg_ref, gt == "bf16")
    assert not dg.view(T, B, 2 * H)[pad].any()
    close(dh0.cpu().numpy().reshape(B, H), dh0_ref, False)
    assert intact(gb, T * B * 2 * H) and intact(eb, B * H)


TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")]


@pytest.mark.parametrize("gt,ht", TYPES)
@pytest.mark.parametrize("T,B,H", [(1, 1, 1), (2, 3, 5), (3, 1, 64), (17, 2, 31), (64, 2, 130), (129, 3, 96),
                                   (500, 1, 257), (1025, 2, 66)])
def test_forward_and_backward(T, B, H, gt, ht):
    check_both(T, B, H, gt, ht, seed=T * 1000 + H)


@pytest.mark.parametrize("gt,ht", TYPES)
@pytest.mark.parametrize("T,H,lengths", [
    (1, 40, [0, 1, 1]), (7, 33, [0, 7, 3, 1, 6]), (100, 64, [100, 0, 1, 99, 64, 65, 63]),
    (700, 34, [0, 0, 0]), (513, 128, [512, 513, 1, 0, 256, 255, 257, 128]),
    (90, 16, [-5, 1000, 2 ** 31 - 1, -2 ** 31]),  # clamped to [0, T]
])
def test_padding_is_neither_read_nor_carried(T, H, lengths, gt, ht):
    check_both(T, len(lengths), H, gt, ht, seed=T + H, lengths=lengths)


def test_infinities_in_padding():
    check_both(70, 4, 36, "f32", "f32", seed=5, lengths=[70, 30, 1, 0], poison=float("inf"))


@pytest.mark.parametrize("use_h0,use_last", [(False, True), (True, False), (False, False)])
def test_optional_arguments(use_h0, use_last):
    check_both(150, 2, 48, "bf16", "f32", seed=9, lengths=[150, 20], use_h0=use_h0, use_last=use_last)


@pytest.mark.parametrize("T,B,H", [(128, 32, 1024), (4096, 1, 128), (16384, 1, 40), (3000, 1, 1024), (40, 300, 8)])
def test_ordinary_and_long(T, B, H):
    check_both(T, B, H, "bf16", "bf16", seed=11)
    check_both(T, B, H, "f32", "bf16", seed=12, lengths=[T - (T * b) // B for b in range(B)])


@pytest.mark.parametrize("gt,ht", TYPES)
@pytest.mark.parametrize("T,B,H,shift", [(70, 3, 67, 0), (70, 2, 67, 1), (41, 1, 129, 1), (33, 2, 66, 1), (65, 3, 1, 1),
                                         (40, 1, 63, 3), (300, 1, 65, 1), (34, 2, 128, 1)])
def test_rows_on_any_element(T, B, H, shift, gt, ht):
    """Tensors that start `shift` elements into a buffer, rows of odd and even
    widths: nothing before or behind an array is written, and its first and
    last words are right."""
    import torch
    g, h0, n, dh, dl = make(T, B, H, gt, ht, seed=T + H)

    def at(t):
        buf = torch.full((t.numel() + shift + 8,), CANARY, dtype=t.dtype, device="cuda")
        buf[shift:shift + t.numel()] = t.reshape(-1).cuda()
        return buf, buf[shift:shift + t.numel()]

    def clean(buf, n):
        return bool((buf[:shift] == buf.new_tensor(CANARY)).all()) and bool((buf[shift + n:] == buf.new_tensor(CANARY)).all())

    gd, dhd = at(g)[1], at(dh)[1]
    hb, h = at(torch.zeros(T, B, H, dtype=tdtype(ht)))
    db, dg = at(torch.zeros(T, B, 2 * H, dtype=tdtype(gt)))
    last, dh0 = torch.empty(B, H, device="cuda"), torch.empty(B, H, device="cuda")
    isam.glr_forward(T, B, H, gd, h0.cuda(), None, h, last)
    isam.glr_backward(T, B, H, gd, h0.cuda(), None, h, dhd, dl.cuda(), dg, dh0)
    isam.sync()
    out, lr = lm_ref.recurrence(f64(g), f64(h0), n)
    close(h.float().cpu().numpy().reshape(T, B, H), out, ht == "bf16")
    close(last.cpu().numpy(), lr, False)
    dref, eref = lm_ref.recurrence_backward(f64(g), f64(h0), n, h.double().cpu().numpy().reshape(T, B, H), f64(dh), f64(dl))
    close(dg.float().cpu().numpy().reshape(T, B, 2 * H), dref, gt == "bf16")
    close(dh0.cpu().numpy(), eref, False)
    assert clean(hb, T * B * H) and clean(db, T * B * 2 * H)


@pytest.mark.parametrize("gt,ht", TYPES)
@pytest.mark.parametrize("T,B,H,lengths", [(16, 3, 65, None), (17, 3, 65, None), (19, 130, 1021, None),
                                           (18, 256, 4096, None), (21, 4, 33000, [21, 0, 1, 9])])
def test_few_steps_and_many_channels(T, B, H, lengths, gt, ht):
    check_both(T, B, H, gt, ht, seed=T + B, lengths=lengths)


@pytest.mark.parametrize("gt,ht", TYPES)
@pytest.mark.parametrize("T,B,H,lengths", [(32, 128, 1024, None), (33, 128, 1024, None), (45, 50, 1001, "ragged"),
                                           (41, 48, 1026, "ragged"), (30, 47, 1021, "ragged"), (25, 1025, 512, "ragged")])
def test_either_side_of_the_choice(T, B, H, lengths, gt, ht):
    check_both(T, B, H, gt, ht, seed=T + H,
               lengths=lengths and [(7 * b) % (T + 1) for b in range(B)])


@pytest.mark.parametrize("T", [3, 40])
def test_gates_beyond_every_exponent(T):
    """z = 0 and z = 1 from gates as large as they get, for few steps and many."""
    import torch
    B, H = 2, 64
    for gate, want in ((-200.0, 3.0), (-float("inf"), 3.0), (200.0, 0.5), (float("inf"), 0.5)):
        g = torch.empty(T, B, 2 * H, device="cuda")
        g[:, :, :H], g[:, :, H:] = gate, 3.0
        h0 = torch.full((B, H), 0.5, device="cuda")
        out, last = torch.empty(T, B, H, device="cuda"), torch.empty(B, H, device="cuda")
        isam.glr_forward(T, B, H, g, h0, None, out, last)
        isam.sync()
        # 1 - z is a product of two numbers good to 2^-22 each.
        assert torch.allclose(out, torch.full_like(out, want), rtol=1e-6, atol=0.0)
        assert torch.allclose(last, torch.full_like(last, want), rtol=1e-6, atol=0.0)


def test_saturated_gates():
    """z = 1 to the last bit: the state stays h0 (what is taken of n, e^-40,
    is below a unit of it); z = 0: the state is the candidate."""
    import torch
    T, B, H = 2000, 1, 64
    g = torch.empty(T, B, 2 * H, device="cuda")
    g[:, :, :H], g[:, :, H:] = 40.0, 3.0
    h0 = torch.linspace(-2, 2, H, device="cuda").view(1, H)
    out, last = torch.empty(T, B, H, device="cuda"), torch.empty(B, H, device="cuda")
    isam.glr_forward(T, B, H, g, h0, None, out, last)
    isam.sync()
    assert (out - h0).abs().max() < 1e-12 and (last - h0).abs().max() < 1e-12
    g[:, :, :H] = -40.0
    g[:, :, H:] = torch.randn(T, B, H, device="cuda")
    isam.glr_forward(T, B, H, g, h0, None, out, last)
    isam.sync()
    assert torch.allclose(out, g[:, :, H:], rtol=1e-6, atol=1e-12)


def test_infinite_gates_and_candidates():
    """g_z = +inf keeps the state (1 - z is exactly 0), -inf replaces it; an
    infinite candidate under a finite gate makes that channel infinite, and
    only that channel."""
    import torch
    T, H = 300, 8
    g = torch.randn(T, 1, 2 * H, device="cuda")
    g[100, 0, 0], g[100, 0, 1], g[100, 0, H + 2] = float("inf"), float("-inf"), float("inf")
    h0 = torch.zeros(1, H, device="cuda")
    out = torch.empty(T, 1, H, device="cuda")
    isam.glr_forward(T, 1, H, g, h0, None, out, None)
    isam.sync()
    assert out[100, 0, 0] == out[99, 0, 0] and out[100, 0, 1] == g[100, 0, H + 1]
    assert torch.isinf(out[100:, 0, 2]).all()
    keep = [c for c in range(H) if c != 2]
    assert torch.isfinite(out[:, 0, keep]).all() and torch.isfinite(out[:100]).all()


def test_gradient_against_differences():
    """Directional derivatives of the 64-bit forward form by central
    differences (error O(eps^2) = 1e-8 of the scale) against the library's
    gradients.  The fp32 gradient's own tolerance, F32 of the largest value in
    each of the n terms of the product, adds up as sqrt(n)."""
    import torch
    T, B, H = 60, 3, 10
    n = np.array([60, 17, 0])
    g, h0, _, dh, dl = make(T, B, H, "f32", "f32", seed=21, lengths=n)
    rng = np.random.default_rng(22)

    def loss(gv, hv):
        out, last = lm_ref.recurrence(gv, hv, n)
        live = (np.arange(T)[:, None] < n[None, :])[:, :, None]
        return float((out * f64(dh) * live).sum() + (last * f64(dl)).sum())

    h = torch.empty(T, B, H, device="cuda")
    ld = torch.from_numpy(n.astype(np.int32)).cuda()
    dg, dh0 = torch.empty(T, B, 2 * H, device="cuda"), torch.empty(B, H, device="cuda")
    isam.glr_forward(T, B, H, g.cuda(), h0.cuda(), ld, h, None)
    isam.glr_backward(T, B, H, g.cuda(), h0.cuda(), ld, h, dh.cuda(), dl.cuda(), dg, dh0)
    isam.sync()
    dg, dh0 = dg.double().cpu().numpy(), dh0.double().cpu().numpy()
    for _ in range(6):
        v, w = rng.standard_normal(g.shape), rng.standard_normal(h0.shape)
        eps = 1e-4
        num = (loss(f64(g) + eps * v, f64(h0) + eps * w) - loss(f64(g) - eps * v, f64(h0) - eps * w)) / (2 * eps)
        got = float((dg * v).sum() + (dh0 * w).sum())
        tol = F32 * np.abs(dg).max() * np.sqrt(v.size) * 4 + 1e-6 * abs(num) + 1e-6
        assert abs(got - num) <= tol, (got, num, tol)


def test_in_place_state_and_chunked_sequences():
    """h_last may be h0, and a sequence run in pieces gives the states of the
    whole (each piece starts from the last one's h_last)."""
    import torch
    T, B, H = 333, 2, 70
    g, h0, _, _, _ = make(T, B, H, "f32", "f32", seed=31)
    g, h0 = g.cuda(), h0.cuda()
    whole, last = torch.empty(T, B, H, device="cuda"), torch.empty(B, H, device="cuda")
    isam.glr_forward(T, B, H, g, h0, None, whole, last)
    state, parts = h0.clone(), torch.empty(T, B, H, device="cuda")
    for a, b in ((0, 1), (1, 130), (130, 332), (332, 333)):
        isam.glr_forward(b - a, B, H, g[a:b], state, None, parts[a:b], state)
    isam.sync()
    tol = F32 * float(whole.abs().max())
    assert (parts - whole).abs().max() <= tol and (state - last).abs().max() <= tol


def test_repeated_calls_give_the_same_bits_on_another_stream():
    import torch
    T, B, H = 2500, 1, 512
    g, h0, _, dh, dl = (t.cuda() if isinstance(t, torch.Tensor) else t for t in make(T, B, H, "bf16", "bf16", seed=41))
    outs = []
    for s in (torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            h, last = torch.empty(T, B, H, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, device="cuda")
            dg, dh0 = torch.empty_like(g), torch.empty(B, H, device="cuda")
            isam.glr_forward(T, B, H, g, h0, None, h, last)
            isam.glr_backward(T, B, H, g, h0, None, h, dh, dl, dg, dh0)
            isam.sync()
        outs.append((h, last, dg, dh0))
    for o in outs[1:]:
        for a, b in zip(outs[0], o):
            assert torch.equal(a, b)


def test_captured_in_a_graph():
    import torch
    T, B, H = 300, 2, 64
    g, h0, _, dh, dl = (t.cuda() if isinstance(t, torch.Tensor) else t for t in make(T, B, H, "f32", "f32", seed=51))
    h, last = torch.empty(T, B, H, device="cuda"), torch.empty(B, H, device="cuda")
    isam.glr_forward(T, B, H, g, h0, None, h, last)
    isam.sync()
    want = h.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        isam.glr_forward(T, B, H, g, h0, None, h, last)
    h.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, want)


def test_offsets_beyond_32_bits():
    """More than 2^31 gate values: the rows behind the 32-bit range are right
    (checked on a few channels, whose states forget what came long before)."""
    import torch
    T, B, H = 540_000, 1, 2048
    assert T * 2 * H > 2 ** 31
    g = torch.empty(T, B, 2 * H, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    g.normal_(generator=gen)
    h = torch.empty(T, B, H, dtype=torch.bfloat16, device="cuda")
    last = torch.empty(B, H, device="cuda")
    isam.glr_forward(T, B, H, g, None, None, h, last)
    dl = torch.randn(B, H, device="cuda")
    dh = h  # any gradient of the right type
    dg, dh0 = torch.empty_like(g), torch.empty(B, H, device="cuda")
    isam.glr_backward(T, B, H, g, None, None, h, dh, dl, dg, dh0)
    isam.sync()
    cols, tail = [0, 1, 1023, 2047], 400
    two = cols + [c + H for c in cols]
    gs = g[-tail:, :, two].double().cpu().numpy()
    hs = h[-tail - 1:, :, cols].double().cpu().numpy()
    n = np.array([tail])
    out, lr = lm_ref.recurrence(gs, hs[0], n)
    close(h[-200:, :, cols].float().cpu().numpy(), out[-200:], True)
    close(last[:, cols].cpu().numpy(), lr, False)
    dref, _ = lm_ref.recurrence_backward(gs, hs[0], n, hs[1:], hs[1:], dl[:, cols].double().cpu().numpy())
    close(dg[-tail:, :, two].float().cpu().numpy(), dref, True)
    head = 300
    gs, hs = g[:head, :, two].double().cpu().numpy(), h[:head, :, cols].double().cpu().numpy()
    n = np.array([head])
    out, _ = lm_ref.recurrence(gs, np.zeros((1, 4)), n)
    close(hs, out, True)


@pytest.mark.parametrize("gt,ht", TYPES)
@pytest.mark.parametrize("B,H,slots,in_place", [(1, 1, 1, True), (5, 33, 9, False), (32, 1024, 64, True),
                                                (300, 66, 301, False), (7, 2560, 7, True)])
def test_step(B, H, slots, in_place, gt, ht):
    import torch
    rng = np.random.default_rng(B + H)
    g = torch.from_numpy(rng.standard_normal((B, 2 * H))).to(tdtype(gt))
    state = torch.from_numpy(rng.standard_normal((slots, H)).astype(np.float32))
    ids = rng.permutation(slots)[:B].astype(np.int32)
    bad = [b for b in range(B) if B > 4 and b % 4 == 1]
    for i, b in enumerate(bad):
        ids[b] = (-1, slots, 2 ** 31 - 1, -2 ** 31)[i % 4]
    ref_h, ref_s = np.zeros((B, H)), f64(state)
    for b in range(B):
        if 0 <= ids[b] < slots:
            z, r = lm_ref.sigmoid(f64(g)[b, :H]), lm_ref.sigmoid(-f64(g)[b, :H])
            ref_h[b] = ref_s[ids[b]] = z * ref_s[ids[b]] + r * f64(g)[b, H:]
    sd = state.cuda()
    buf, new = guarded((slots, H), torch.float32)
    new.copy_(state.reshape(-1))
    new = sd.view(-1) if in_place else new
    hb, h = guarded((B, H), tdtype(ht))
    isam.glr_step(B, H, slots, g.cuda(), torch.from_numpy(ids).cuda(), sd, new, h)
    isam.sync()
    close(h.float().cpu().numpy().reshape(B, H), ref_h, ht == "bf16")
    close(new.cpu().numpy().reshape(slots, H), ref_s, False)
    rest = sorted(set(range(slots)) - {int(i) for i in ids if 0 <= i < slots})
    assert torch.equal(new.cpu().view(slots, H)[rest], state[rest])
    if not in_place:
        assert torch.equal(sd.cpu(), state)
    assert intact(buf, slots * H) and intact(hb, B * H)


def test_step_equals_a_sequence_of_one():
    import torch
    B, H = 9, 130
    g, h0, _, _, _ = make(1, B, H, "bf16", "f32", seed=61)
    out, last = torch.empty(1, B, H, device="cuda"), torch.empty(B, H, device="cuda")
    isam.glr_forward(1, B, H, g.cuda(), h0.cuda(), None, out, last)
    state, h = h0.cuda(), torch.empty(B, H, device="cuda")
    isam.glr_step(B, H, B, g.cuda(), None, state, state, h)
    isam.sync()
    tol = F32 * float(last.abs().max())
    assert (h - out[0]).abs().max() <= tol and (state - last).abs().max() <= tol


# Rows by TMA, as lane words and as covering words (bf16 gates), and walked.
FORMS = [(70, 3, 128), (70, 3, 66), (70, 3, 67), (9, 3, 66)]


@pytest.mark.parametrize("gt,ht", TYPES)
@pytest.mark.parametrize("T,B,H", FORMS)
@pytest.mark.parametrize("lengths", [None, [70, 0, 33]])
def test_no_gradient_of_the_states(T, B, H, lengths, gt, ht):
    """dh_out = NULL stands for zeros: the same bits, from dh_last alone."""
    import torch
    g, h0, _, _, dl = make(T, B, H, gt, ht, seed=T + H)
    g, h0, dl = g.cuda(), h0.cuda(), dl.cuda()
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    h = torch.empty(T, B, H, dtype=tdtype(ht), device="cuda")
    isam.glr_forward(T, B, H, g, h0, n, h)
    got = []
    for dh in (torch.zeros_like(h), None):
        gb, dg = guarded((T, B, 2 * H), tdtype(gt))
        eb, dh0 = guarded((B, H), torch.float32)
        isam.glr_backward(T, B, H, g, h0, n, h, dh, dl, dg, dh0)
        isam.sync()
        assert intact(gb, T * B * 2 * H) and intact(eb, B * H)
        assert torch.isfinite(dg).all() and dg.any()
        got.append((dg, dh0))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("gt,ht", TYPES)
@pytest.mark.parametrize("T,B,H", FORMS + [(1536, 5, 2048), (1536, 5, 2046), (1500, 3, 1021)])
@pytest.mark.parametrize("ragged", [False, True])
def test_states_in_place_give_the_same_bits(T, B, H, ragged, gt, ht):
    """h_last = h0 and dh0 = dh_last, also where a cluster of several CTAs takes
    several groups of channels one after another (5 x 2048)."""
    import torch
    g, h0, _, dh, dl = make(T, B, H, gt, ht, seed=T + H)
    g, h0, dh, dl = g.cuda(), h0.cuda(), dh.cuda(), dl.cuda()
    n = torch.tensor([(T * b) // (B - 1) for b in range(B)], dtype=torch.int32, device="cuda") if ragged else None
    out = []
    for in_place in (False, True):
        h = torch.empty(T, B, H, dtype=tdtype(ht), device="cuda")
        state, e = h0.clone(), dl.clone()
        last = state if in_place else torch.empty_like(state)
        dh0 = e if in_place else torch.empty_like(e)
        isam.glr_forward(T, B, H, g, state, n, h, last)
        dg = torch.empty_like(g)
        isam.glr_backward(T, B, H, g, h0, n, h, dh, e, dg, dh0)
        isam.sync()
        out.append((h, last, dg, dh0))
    assert all(torch.equal(a, b) for a, b in zip(*out))
