"""The 4-bit few-token product and its packing on the GPU against the
definition in 64 bits.

Tolerance.  Products of bf16 x and (q - 8) are exact in fp32.  A sum of K of
them, multiplied by scales, takes at most K/16 + 32 additions one after
another (the tensor cores add 16 products at a time); each loses at most 2^-22
of the sum of magnitudes (truncation), so a result is within
(K/16 + 32) 2^-22 sum |x w| of the true one.  Integer x with power-of-two
scales must be exact."""
import numpy as np
import pytest

import lm_ref
from gpu_util import Guarded
from paper_1810_09958_gb300 import isam

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import torch
    from paper_1810_09958_gb300 import build
    build.build()
    isam.load()
    torch.cuda.set_device(0)
    yield
    isam.sync()


def weights(N, K, group, seed, exact=False):
    import torch
    rng = np.random.default_rng(seed)
    q = rng.integers(0, 16, (N, K)).astype(np.uint8)
    groups = -(-K // group)
    s = 2.0 ** rng.integers(-3, 4, (N, groups)) if exact else rng.uniform(0.002, 0.02, (N, groups))
    return q, torch.from_numpy(s).bfloat16()


def packed(q, s, group):
    import torch
    N, K = q.shape
    tiled = torch.full((isam.w4_tiled_bytes(N, K),), 0xAA, dtype=torch.uint8, device="cuda")
    ts = torch.full((isam.w4_tiled_scales(N, K, group),), float("nan"), dtype=torch.bfloat16, device="cuda")
    isam.w4_pack(N, K, group, torch.from_numpy(lm_ref.pack_rows(q)).cuda(), s.cuda(), tiled, ts)
    return tiled, ts


def inputs(M, K, seed, exact=False):
    import torch
    rng = np.random.default_rng(seed + 1)
    x = rng.integers(-4, 5, (M, K)).astype(np.float64) if exact else rng.standard_normal((M, K))
    return torch.from_numpy(x).bfloat16()


def check(M, N, K, group, seed, exact=False):
    q, s = weights(N, K, group, seed, exact)
    x = inputs(M, K, seed, exact)
    tiled, ts = packed(q, s, group)
    y = Guarded(M * N, np.full(M * N, np.nan))
    isam.gemv_w4(M, N, K, group, x.cuda(), tiled, ts, y.t)
    isam.sync()
    w = lm_ref.dequantised(q, s.double().numpy(), group)
    ref = x.double().numpy() @ w.T
    got = y.numpy().astype(np.float64).reshape(M, N)
    if exact:
        assert np.array_equal(got, ref)
    else:
        tol = (K / 16 + 32) * 2.0 ** -22 * (np.abs(x.double().numpy()) @ np.abs(w).T)
        assert (np.abs(got - ref) <= tol).all()
    assert y.guards_intact()


@pytest.mark.parametrize("N,K,group", [(1, 8, 32), (16, 128, 128), (17, 136, 32), (33, 200, 64), (5, 1000, 128)])
def test_packed_order_is_the_documented_one(N, K, group):
    q, s = weights(N, K, group, seed=N + K)
    tiled, ts = packed(q, s, group)
    nb, kb, per = -(-N // 16), -(-K // 128), 128 // group
    words = tiled.cpu().numpy().view("<u4").reshape(nb, kb, 2, 8, 4, 4)
    for at in np.ndindex(words.shape):
        b, k, half, r, t, j = at
        assert int(words[at]) == lm_ref.tiled_word(q, b, k, half, r, t, j), at
    sc = ts.float().cpu().numpy().reshape(nb, kb, 16, per)
    full = np.zeros((nb * 16, kb * per), np.float32)
    full[:N, : s.shape[1]] = s.float().numpy()
    assert np.array_equal(sc, full.reshape(nb, 16, kb, per).transpose(0, 2, 1, 3))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [1, 2, 3, 7, 8, 9, 16, 17, 24, 25, 32])
def test_tokens(M, group):
    check(M, 72, 640, group, seed=M)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 8), (1, 4096), (15, 16), (16, 24), (17, 128), (31, 136), (33, 2000), (100, 1032),
                                 (2049, 256), (513, 8192), (4096, 4096)])
@pytest.mark.parametrize("M", [1, 5])
def test_sizes(M, N, K, group):
    check(M, N, K, group, seed=N + K)


@pytest.mark.parametrize("M,N,K,group", [(8, 40, 16384, 32), (9, 50, 8200, 64), (16, 33, 9000, 32), (17, 65, 4104, 128),
                                         (32, 100, 5000, 32), (1, 2500, 264, 64), (3, 4900, 40, 32), (20, 2600, 136, 128)])
def test_x_that_fits_and_x_that_does_not(M, N, K, group):
    """x beside the ring in shared memory, and x too large for it; teams of one,
    two, four and eight warps."""
    check(M, N, K, group, seed=M + N + K)


@pytest.mark.parametrize("M,N,K,group", [(1, 7600, 136, 32), (8, 5200, 1544, 128), (13, 5200, 4104, 64),
                                         (16, 5000, 4096, 64), (16, 7500, 200, 32), (20, 5000, 4000, 32),
                                         (32, 7400, 1000, 128), (32, 5000, 2048, 64), (29, 5100, 3080, 128)])
def test_several_groups_of_rows_a_team(M, N, K, group):
    check(M, N, K, group, seed=N + K)


@pytest.mark.parametrize("M,N,K,group", [(1, 160, 1024, 32), (8, 1001, 520, 64), (32, 64, 2048, 128), (3, 7, 40, 32)])
def test_integer_data_is_exact(M, N, K, group):
    check(M, N, K, group, seed=77, exact=True)


def test_every_code_in_every_place():
    """A unit x picks out each k in turn: y is the weight itself."""
    import torch
    N, K, group = 16, 256, 32
    q = ((np.arange(N)[:, None] * 7 + np.arange(K)[None, :]) % 16).astype(np.uint8)
    s = torch.from_numpy(2.0 ** (np.arange(N * 8).reshape(N, 8) % 5 - 2.0)).bfloat16()
    tiled, ts = packed(q, s, group)
    w = lm_ref.dequantised(q, s.double().numpy(), group)
    y = torch.empty(32 * N, device="cuda")
    for k0 in range(0, K, 32):
        x = torch.zeros(32, K)
        x[torch.arange(32), k0 + torch.arange(32)] = 1
        isam.gemv_w4(32, N, K, group, x.bfloat16().cuda(), tiled, ts, y)
        isam.sync()
        assert np.array_equal(y.cpu().numpy().reshape(32, N), w[:, k0:k0 + 32].T)


def test_infinite_x_reaches_its_token_alone():
    import torch
    M, N, K, group = 4, 48, 256, 64
    q, s = weights(N, K, group, seed=3)
    tiled, ts = packed(q, s, group)
    x = inputs(M, K, 3)
    y0, y1 = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda")
    isam.gemv_w4(M, N, K, group, x.cuda(), tiled, ts, y0)
    x[2, 100] = float("inf")
    isam.gemv_w4(M, N, K, group, x.cuda(), tiled, ts, y1)
    isam.sync()
    rows = [0, 1, 3]
    assert torch.equal(y0[rows], y1[rows]) and not torch.isfinite(y1[2]).any()


def test_same_bits_on_another_stream():
    import torch
    q, s = weights(500, 4096, 32, seed=4)
    tiled, ts = packed(q, s, 32)
    x = inputs(6, 4096, 4).cuda()
    isam.sync()
    outs = []
    for st in (torch.cuda.current_stream(), torch.cuda.Stream()):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            y = torch.empty(6, 500, device="cuda")
            isam.gemv_w4(6, 500, 4096, 32, x, tiled, ts, y)
            isam.sync()
            outs.append(y)
    assert torch.equal(outs[0], outs[1])


def test_weights_beyond_32_bits():
    """More than 2^32 codes: the last rows are right."""
    import torch
    N, K, group = 300_000, 16_384, 128
    assert N * K > 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
    scales = torch.rand(N, K // group, device="cuda", generator=gen).mul_(0.01).bfloat16()
    tiled = torch.empty(isam.w4_tiled_bytes(N, K), dtype=torch.uint8, device="cuda")
    ts = torch.empty(isam.w4_tiled_scales(N, K, group), dtype=torch.bfloat16, device="cuda")
    isam.w4_pack(N, K, group, codes, scales, tiled, ts)
    x = inputs(2, K, 5)
    y = torch.empty(2, N, device="cuda")
    isam.gemv_w4(2, N, K, group, x.cuda(), tiled, ts, y)
    isam.sync()
    c = codes[-64:].cpu().numpy()
    q = np.empty((64, K), np.uint8)
    q[:, 0::2], q[:, 1::2] = c & 15, c >> 4
    w = lm_ref.dequantised(q, scales[-64:].double().cpu().numpy(), group)
    tol = (K / 16 + 32) * 2.0 ** -22 * (np.abs(x.double().numpy()) @ np.abs(w).T)
    assert (np.abs(y[:, -64:].double().cpu().numpy() - x.double().numpy() @ w.T) <= tol).all()


@pytest.mark.parametrize("M,K", [(2, 2 ** 30 - 128), (2, 2 ** 30 - 8), (1, 2 ** 30), (2, 2 ** 30 + 264), (1, 2 ** 31 - 8)])
def test_rows_of_x_beyond_32_bits(M, K):
    """Rows of x of 2 and 4 GB: their size passes 31 and 32 bits.  x is zero but
    in a few places, integers there, so that results are exact."""
    import torch
    N, group = 3, 128
    gen = torch.Generator(device="cuda").manual_seed(K % 1000)
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
    scales = torch.randint(0, 4, (N, -(-K // group)), device="cuda", generator=gen).sub_(2).float().exp2_().bfloat16()
    tiled = torch.empty(isam.w4_tiled_bytes(N, K), dtype=torch.uint8, device="cuda")
    ts = torch.empty(isam.w4_tiled_scales(N, K, group), dtype=torch.bfloat16, device="cuda")
    isam.w4_pack(N, K, group, codes, scales, tiled, ts)
    at = [0, 1, 129, K // 3, K // 2 - 1, K // 2, K - 130, K - 2, K - 1]
    at += [k for k in (2 ** 29 - 1, 2 ** 29, 2 ** 30 - 1, 2 ** 30) if k < K and k not in at]
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    v = np.arange(1, len(at) + 1) * (1 + np.arange(M)[:, None])
    x[:, at] = torch.from_numpy(v.astype(np.float32)).bfloat16().cuda()
    y = Guarded(M * N, np.full(M * N, np.nan))
    isam.gemv_w4(M, N, K, group, x, tiled, ts, y.t)
    isam.sync()
    k = torch.tensor(at, device="cuda")
    pair = codes[:, k // 2].cpu().numpy()
    q = np.where(np.array(at) % 2 == 0, pair & 15, pair >> 4).astype(np.float64)
    w = (q - 8) * scales[:, k // group].double().cpu().numpy()
    assert np.array_equal(y.numpy().astype(np.float64).reshape(M, N), v @ w.T)
    assert y.guards_intact()
