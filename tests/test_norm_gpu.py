"""Root-mean-square norm with the residual's addition, its block-scaled output
and its backward pass, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_1810_09958_gb300 import isam

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
# Relative error of y in 32 bits: up to 32 squares a thread, 5 folds and 32 warps (69 half steps of the
# mean, half of that of its root), rsqrtf's two steps, and a rounding each of r, r k and the product.
Y32 = 48 * ref.U


def tensor(rng, shape, kind, scale=1.0):
    """On the device, and its exact values."""
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(TYPES[kind]).cuda()
    return t, t.double().cpu().numpy()


def guarded(n, dtype):
    """n elements at an odd place among guard elements: (whole, part)."""
    whole = torch.full((n + 64,), 77, dtype=torch.uint8, device="cuda").repeat_interleave(dtype.itemsize).view(dtype)
    return whole, whole[32: 32 + n]


def intact(whole, n):
    b = whole.view(torch.uint8).view(-1, whole.dtype.itemsize)
    return bool((b[:32] == 77).all() and (b[32 + n:] == 77).all())


SIZES = [(1, 1), (1, 7), (3, 8), (2, 31), (5, 33), (1, 255), (7, 256), (2, 257), (3, 1001), (1, 1024), (2, 4096),
         (1, 5120), (3, 8191), (2, 8192), (1, 8200), (2, 9999), (1, 16384), (2, 32767), (1, 32768), (700, 72)]


@pytest.mark.parametrize("x_kind,r_kind,y_kind", [("fp32", "bf16", "bf16"), ("bf16", "bf16", "bf16"),
                                                  ("bf16", "fp32", "fp32"), ("fp32", "fp32", "bf16")])
@pytest.mark.parametrize("T,D", SIZES)
def test_forward(T, D, x_kind, r_kind, y_kind):
    rng = np.random.default_rng(T * 40000 + D)
    x, x64 = tensor(rng, (T, D), x_kind)
    res, res64 = tensor(rng, (T, D), r_kind, 3.0)
    w, w64 = tensor(rng, (D,), "fp32")
    whole_r, res_out = guarded(T * D, TYPES[r_kind])
    whole_y, y = guarded(T * D, TYPES[y_kind])
    isam.rms_norm_forward(T, D, x, res, res_out, w, EPS, y)
    isam.sync()
    want, r = ref.norm(x64, res64, w64, EPS)
    assert (np.abs(y.view(T, D).double().cpu().numpy() - want) <= (Y32 + ref.HALF[y_kind]) * np.abs(want) + 1e-37).all()
    assert (np.abs(res_out.view(T, D).double().cpu().numpy() - r) <= (ref.U + ref.HALF[r_kind]) * np.abs(r)).all()
    assert intact(whole_r, T * D) and intact(whole_y, T * D)


@pytest.mark.parametrize("T,D", [(1, 32), (4, 1000), (3, 4096), (2, 8193)])
def test_forward_without_a_residual_and_in_place(T, D):
    rng = np.random.default_rng(D)
    x, x64 = tensor(rng, (T, D), "bf16")
    w, w64 = tensor(rng, (D,), "fp32")
    y = torch.empty(T, D, device="cuda")
    isam.rms_norm_forward(T, D, x, None, None, w, EPS, y)
    want, _ = ref.norm(x64, None, w64, EPS)
    assert (np.abs(y.double().cpu().numpy() - want) <= (Y32 + ref.U) * np.abs(want) + 1e-37).all()
    copy = torch.empty(T, D, device="cuda")
    isam.rms_norm_forward(T, D, x, None, copy, w, EPS, y)  # r itself wanted
    assert torch.equal(copy, x.float())
    res, res64 = tensor(rng, (T, D), "fp32", 2.0)
    isam.rms_norm_forward(T, D, x, res, res, w, EPS, y)  # in place
    want, r = ref.norm(x64, res64, w64, EPS)
    assert (np.abs(y.double().cpu().numpy() - want) <= (Y32 + ref.U) * np.abs(want) + 1e-37).all()
    assert (np.abs(res.double().cpu().numpy() - r) <= ref.U * np.abs(r)).all()


def check_mx(y8, scales, want):
    T, D = want.shape
    atoms = -(-D // 128)
    byte = scales.cpu().numpy().reshape(atoms, T, 4).transpose(1, 0, 2).reshape(T, atoms * 4).astype(np.int64)
    full = np.zeros((T, atoms * 128))
    full[:, :D] = want
    top = np.abs(full.reshape(T, atoms * 4, 32)).max(axis=2)
    lo = np.ceil(np.log2(np.maximum(top * (1 - Y32), 1e-300) / 448)).clip(-127, 127) + 127
    hi = np.ceil(np.log2(np.maximum(top * (1 + Y32), 1e-300) / 448)).clip(-127, 127) + 127
    assert ((byte >= lo) & (byte <= hi)).all()
    s = np.repeat(2.0 ** (byte - 127.0), 32, axis=1)[:, :D]
    got = ref.e4m3(y8.cpu().numpy().reshape(T, D)) * s
    # Half a step of E4M3: 2^-4 of a normal value, 2^-10 of the scale below.
    assert (np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s) + Y32 * np.abs(want)).all()


@pytest.mark.parametrize("x_kind,r_kind", [("fp32", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("T,D", SIZES)
def test_forward_block_scaled(T, D, x_kind, r_kind):
    rng = np.random.default_rng(T * 40000 + D)
    x, x64 = tensor(rng, (T, D), x_kind)
    res, res64 = tensor(rng, (T, D), r_kind)
    wide = np.exp2(rng.integers(-20, 12, D)).astype(np.float32)  # blocks of very different size
    w = torch.from_numpy(wide).cuda()
    whole8, y8 = guarded(T * D, torch.uint8)
    n = -(-D // 128) * T * 4
    whole_s, scales = guarded(n, torch.uint8)
    isam.rms_norm_forward(T, D, x, res, None, w, EPS, None, y8, scales)
    isam.sync()
    check_mx(y8, scales, ref.norm(x64, res64, wide.astype(np.float64), EPS)[0])
    assert intact(whole8, T * D) and intact(whole_s, n)


@pytest.mark.parametrize("D", [128, 131])
def test_block_scales_of_zeros_nan_and_borders(D):
    T = 5
    x = torch.zeros(T, D, device="cuda")
    x[1, 3] = float("nan")
    x[2, 40] = float("inf")
    x[3] = 1.0  # every y is w
    w = torch.ones(D, device="cuda")
    w[:32], w[32:64], w[64:96] = 448.0, 449.0, 0.4375  # 448 2^0; above it; 448 2^-10
    y8, scales = torch.empty(T, D, dtype=torch.uint8, device="cuda"), torch.empty(-(-D // 128), T, 4, dtype=torch.uint8, device="cuda")
    isam.rms_norm_forward(T, D, x, None, None, w, 1e-5, None, y8, scales)
    v, s = y8.cpu().numpy(), scales.cpu().numpy()
    assert (v[0] == 0).all() and (s[:, 0] == 0).all()           # zeros
    assert (v[1] == 0x7f).all() and (s[0, 1] == 255).all()      # a NaN in a row is in all of its mean
    assert (v[2, 32:64] == 0x7f).all() and s[0, 2, 1] == 255    # inf / inf; the others are 0
    assert (v[2, :32] == 0).all() and s[0, 2, 0] == 0
    x[3] = 1.0
    isam.rms_norm_forward(1, D, x[3], None, None, w, 0.0, None, y8[:1], scales.view(-1)[: -(-D // 128) * 4])
    s = scales.view(-1).cpu().numpy()
    assert s[0] == 127 and s[1] == 128 and s[2] == 117
    assert (y8[0, :32].cpu().numpy() == 0x7e).all()             # 448 itself


def test_block_scaled_output_is_the_block_scaled_products_operand():
    T, D, N = 70, 384, 48
    rng = np.random.default_rng(3)
    x, x64 = tensor(rng, (T, D), "fp32")
    w, w64 = tensor(rng, (D,), "fp32")
    y8, sa = torch.empty(T, D, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(3 * T * 4, dtype=torch.uint8, device="cuda")
    b8, sb = torch.empty(N, D, dtype=torch.uint8, device="cuda"), torch.empty(3 * N * 4, dtype=torch.uint8, device="cuda")
    weight, weight64 = tensor(rng, (N, D), "fp32")
    isam.rms_norm_forward(T, D, x, None, None, w, EPS, None, y8, sa)
    isam.rms_norm_forward(N, D, weight, None, None, torch.ones(D, device="cuda"), EPS, None, b8, sb)
    C = torch.empty(T, N, device="cuda")
    isam.gemm_mxfp8(T, N, D, 1.0, y8, sa, b8, sb, 0.0, C)
    isam.sync()

    def values(v, s, rows):
        byte = s.cpu().numpy().reshape(3, rows, 4).transpose(1, 0, 2).reshape(rows, 12)
        return ref.e4m3(v.view(torch.uint8).cpu().numpy()) * np.repeat(2.0 ** (byte - 127.0), 32, axis=1)

    a, b = values(y8, sa, T), values(b8, sb, N)
    assert (np.abs(C.double().cpu().numpy() - a @ b.T) <= (D + 2) * ref.U * (np.abs(a) @ np.abs(b).T)).all()


@pytest.mark.parametrize("r_kind,g_kind", [("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("T,D", SIZES + [(2000, 64), (1300, 520), (400, 4104), (320, 12296)])
def test_backward(T, D, r_kind, g_kind):
    rng = np.random.default_rng(T * 40000 + D)
    r, r64 = tensor(rng, (T, D), r_kind, 2.0)
    w, w64 = tensor(rng, (D,), "fp32")
    dy, dy64 = tensor(rng, (T, D), g_kind)
    dres, dres64 = tensor(rng, (T, D), g_kind)
    whole, dx = guarded(T * D, TYPES[g_kind])
    whole_w, dw = guarded(D, torch.float32)
    isam.rms_norm_backward(T, D, r, w, EPS, dy, dres, dx, dw)
    isam.sync()
    want, want_w, size, size_w = ref.norm_backward(r64, w64, EPS, dy64, dres64)
    # k and both means to 48 half steps each (as Y32), four products and a sum; then the type's own rounding.
    bound = 104 * ref.U * size + ref.HALF[g_kind] * np.abs(want) + 1e-37
    assert (np.abs(dx.view(T, D).double().cpu().numpy() - want) <= bound).all()
    # n to 48 half steps; a thread adds at most T / 152 rows, then teams (16), CTAs in fives and 32 by folds.
    assert (np.abs(dw.double().cpu().numpy() - want_w) <= (48 + T / 152 + 16 + 10 + 5 + 4) * ref.U * size_w + 1e-37).all()
    assert intact(whole, T * D) and intact(whole_w, D)


def test_backward_parts_by_themselves_and_in_place():
    T, D = 37, 520
    rng = np.random.default_rng(4)
    r, _ = tensor(rng, (T, D), "bf16")
    w, _ = tensor(rng, (D,), "fp32")
    dy, _ = tensor(rng, (T, D), "bf16")
    dres, _ = tensor(rng, (T, D), "bf16")
    dx, dw = torch.empty_like(dy), torch.empty(D, device="cuda")
    isam.rms_norm_backward(T, D, r, w, EPS, dy, dres, dx, dw)
    only_x, only_w = torch.empty_like(dx), torch.empty_like(dw)
    isam.rms_norm_backward(T, D, r, w, EPS, dy, dres, only_x, None)
    ws = torch.empty(isam.rms_norm_backward_workspace(T, D), dtype=torch.uint8, device="cuda")
    isam.rms_norm_backward(T, D, r, w, EPS, dy, None, None, only_w, ws)
    assert torch.equal(only_x, dx) and torch.equal(only_w, dw)
    for place in (dres.clone(), dy.clone()):
        same = place
        isam.rms_norm_backward(T, D, r, w, EPS, same if torch.equal(same, dy) else dy,
                               same if torch.equal(same, dres) else dres, same, None)
        assert torch.equal(same, dx)


def test_backward_against_differences():
    """Central differences of the 64-bit forward form in a random direction."""
    T, D = 6, 72
    rng = np.random.default_rng(5)
    r, r64 = tensor(rng, (T, D), "fp32")
    w, w64 = tensor(rng, (D,), "fp32")
    dy, dy64 = tensor(rng, (T, D), "fp32")
    dx, dw = torch.empty(T, D, device="cuda"), torch.empty(D, device="cuda")
    isam.rms_norm_backward(T, D, r, w, EPS, dy, None, dx, dw)
    vr, vw, h = rng.standard_normal((T, D)), rng.standard_normal(D), 1e-5
    loss = lambda a, b: (ref.norm(a, None, b, EPS)[0] * dy64).sum()
    by_r = (loss(r64 + h * vr, w64) - loss(r64 - h * vr, w64)) / (2 * h)
    by_w = (loss(r64, w64 + h * vw) - loss(r64, w64 - h * vw)) / (2 * h)
    # Differences are off by h^2 times third derivatives (of order 100 here) and 1e-16 / h; dx and dw by 32 bits.
    assert abs((dx.double().cpu().numpy() * vr).sum() - by_r) <= 1e-4 * np.abs(dx.double().cpu().numpy() * vr).sum()
    assert abs((dw.double().cpu().numpy() * vw).sum() - by_w) <= 1e-4 * np.abs(dw.double().cpu().numpy() * vw).sum()


def test_a_captured_pass_replays_beside_eager_calls():
    T, D = 64, 1024
    rng = np.random.default_rng(6)
    x, _ = tensor(rng, (T, D), "fp32")
    w, _ = tensor(rng, (D,), "fp32")
    res = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    y, y2 = torch.empty(T, D, device="cuda"), torch.empty(T, D, device="cuda")
    r = torch.empty_like(res)
    dx, dw = torch.empty(T, D, device="cuda"), torch.empty(D, device="cuda")

    def step(out, ddx, ddw):
        isam.rms_norm_forward(T, D, x, res, r, w, EPS, out)
        isam.rms_norm_backward(T, D, r, w, EPS, out, None, ddx, ddw)

    step(y, dx, dw)
    graph = torch.cuda.CUDAGraph()
    dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    with torch.cuda.graph(graph):
        step(y2, dx2, dw2)
    x.mul_(2.0)
    graph.replay()
    step(y, dx, dw)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_many_rows_past_32_bits():
    """Row offsets above 2^31 elements: the last rows are as a small call's."""
    T, D = 70001, 32768
    if torch.cuda.mem_get_info()[0] < 16e9:
        pytest.skip("needs 16 GB")
    x = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
    x[-3:].normal_()
    x[:-3] = 0.0
    w = torch.ones(D, device="cuda")
    y = torch.empty_like(x)
    isam.rms_norm_forward(T, D, x, None, None, w, EPS, y)
    few = torch.empty(3, D, dtype=torch.bfloat16, device="cuda")
    isam.rms_norm_forward(3, D, x[-3:].clone(), None, None, w, EPS, few)
    assert torch.equal(y[-3:], few) and not y[:3].any()
