"""Dense products at the ends of float32's range: infinities, NaN and values above the largest bfloat16 number, in every kernel size (needs a GPU)."""
import numpy as np
import pytest

from block_util import U32, UBF, dev, empty, rounded
from oracle import block as ob

pytestmark = pytest.mark.gpu
ACT = {"none": 0, "silu": 1}
FAR = float(np.finfo(np.float32).max)     # above the largest bfloat16 number, 3.39e38
# 32 x 32, 64 x 64, 128 x 128 with W packed (4 x 10 tiles of 128 and more rows, or an even share of both)
SIZES = [(33, 70, 65), (1000, 300, 301), (1000, 650, 650), (4200, 1030, 1027)]


def _same(name, got, want, mag, steps, dtype):
    """Infinities and NaN where the definition has them, the rest within `steps` half-steps of float32 of `mag` and one of its own type."""
    got = got.double().cpu().numpy().reshape(want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: {(np.isnan(got) != np.isnan(want)).sum()} differ in being no number"
    far = np.isinf(want)
    assert np.array_equal(got[far], want[far]) and not np.isinf(got[~far]).any(), f"{name}: infinities"
    ok = np.isfinite(want)
    tol = steps * U32 * mag[ok] + (UBF if dtype == "bf16" else U32) * (np.abs(want[ok]) + steps * U32 * mag[ok]) + 1e-37
    over = np.abs(got[ok] - want[ok]) / tol
    assert over.max(initial=0.0) <= 1.0, f"{name}: {over.max():.3g} of what is allowed"


def _products(x, W):
    """The product and its sum of magnitudes; both as float64 has them, with infinities."""
    with np.errstate(all="ignore"):
        return x @ W, np.abs(x) @ np.abs(W)


def _operands(M, K, N, dtype, seed):
    rng = np.random.default_rng(seed + M)
    x, W = rounded(rng.standard_normal((M, K)), dtype), rounded(rng.standard_normal((K, N)) * 0.1, dtype)
    W[np.abs(W) > 0.4] = 0.25     # (so that a far value times one of them is in the range)
    W[W == 0] = 0.125
    x[x == 0] = 1.0
    return rng, x, W


@pytest.mark.parametrize("M,K,N", SIZES)
def test_forward(M, K, N):
    import torch
    from paper_2506_21788_amd import binding as B
    print("dense range forward", M, K, N, flush=True)
    _, x, W = _operands(M, K, N, "f32", 1)
    x[1, 2], x[2, 3], x[3, 4], x[4, 0], x[4, K - 1] = np.inf, -FAR, np.nan, np.inf, -np.inf
    x[M - 1, K - 1], x[5, 5] = -np.inf, 3.4e38
    W[7, N - 1], W[8, 9], W[9, 10] = np.inf, -np.inf, 3.4e38
    x[:, 9] = np.clip(x[:, 9], -0.5, 0.5)
    want, mag = _products(x, W)
    b = np.full(N, 0.5)
    want = want + b
    ws_b, saved_b = B.dense_workspace_bytes(M, K, N, 0, B.F32)
    ws = torch.empty(max(ws_b, 16), dtype=torch.uint8, device="cuda")
    y = empty((M, N))
    B.dense_fwd(M, K, N, 0, B.F32, dev(x), dev(W), dev(b), None, y, None, ws)
    torch.cuda.synchronize()
    assert np.isinf(want).sum() > M and np.isnan(want).any()
    _same("y", y, want, mag + 0.5, K + 8, "f32")


@pytest.mark.parametrize("dtype,act", [("f32", "none"), ("f32", "silu"), ("bf16", "silu"), ("bf16", "none")])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_reverse(M, K, N, dtype, act):
    import torch
    from paper_2506_21788_amd import binding as B
    print("dense range reverse", M, K, N, dtype, act, flush=True)
    rng, x, W = _operands(M, K, N, dtype, 2)
    code = B.BF16 if dtype == "bf16" else B.F32
    b = np.zeros(N)
    g = rounded(rng.standard_normal((M, N)), dtype)
    g[g == 0] = 1.0
    g[1, 2], g[2, 3], g[M - 1, N - 1] = np.inf, np.nan, -np.inf
    if dtype == "f32":
        g[3, 4] = -FAR
        x[3] *= 0.1
    # (a weight may be infinite where the reverse pass reads it: the forward pass of these inputs is that of the finite one)
    ws_b, saved_b = B.dense_workspace_bytes(M, K, N, ACT[act], code)
    ws, saved = (torch.empty(max(k, 16), dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    y, g_x, gW, g_b = empty((M, N), dtype), empty((M, K), dtype), empty((K, N)), empty(N)
    dx, dW, db, dg = dev(x, dtype), dev(W, dtype), dev(b), dev(g, dtype)
    B.dense_fwd(M, K, N, ACT[act], code, dx, dW, db, None, y, saved, ws)
    B.dense_bwd(M, K, N, ACT[act], code, dx, dW, saved, dg, g_x, gW, g_b, ws)
    torch.cuda.synchronize()
    z, zm = _products(x, W)
    _, d = ob.activation(z, act)
    with np.errstate(all="ignore"):
        gz = g * d
        w_gb = gz.sum(0)
    w_gx, m_gx = _products(gz, W.T)
    w_gW, m_gW = _products(x.T, gz)
    # act' off by 0.8 of z's error and 16 half-steps of its own: relative to |g|, not to |g act'|
    slack = 0.8 * (K + 8) * zm + 16 * (1.0 + np.abs(z)) if act != "none" else np.zeros_like(z)
    own = np.where(np.isfinite(g), np.abs(g), 0.0) * slack
    two = 2.0 ** -16 / U32 if dtype == "bf16" and act != "none" else 0.0     # g_z as two bf16 terms
    s_gx, s_gW = N + 8 + two, M + 8 + two
    assert np.isinf(w_gx).sum() >= K and np.isinf(w_gW).sum() >= K
    _same("g_x", g_x, w_gx, m_gx + own @ np.abs(W).T / s_gx, s_gx, dtype)
    _same("gW", gW, w_gW, m_gW + np.abs(x).T @ own / s_gW, s_gW, "f32")
    _same("g_b", g_b, w_gb, np.abs(np.where(np.isfinite(gz), gz, 0.0)).sum(0) + own.sum(0) / (M + 8), M + 8, "f32")


def test_range_below_which_places_are_lost():
    """Operands keep their 24 bits down to 2^-110; below, what is smaller than 2^-134 of them is lost."""
    import torch
    from paper_2506_21788_amd import binding as B
    rng = np.random.default_rng(3)
    m = 1.0 + rng.random(64)
    for e in (-100, -110, -118, -126):
        x = rounded(m * 2.0 ** e, "f32")[:, None]
        y = empty((64, 1))
        B.dense_fwd(64, 1, 1, 0, B.F32, dev(x), torch.full((1, 1), 2.0 ** 100, device="cuda"), None, None, y, None, None)
        off = np.abs(y.double().cpu().numpy() * 2.0 ** -100 - x)
        assert (off <= 2 * U32 * np.abs(x) + (2.0 ** -134 if e < -110 else 0.0)).all(), e
