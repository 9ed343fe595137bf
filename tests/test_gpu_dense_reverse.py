"""Reverse products of the dense call: every kernel size with several slices of the contraction, and how many bits g_z keeps (needs a GPU)."""
import numpy as np
import pytest

from block_util import U32, close, dev, empty, room, rounded, untouched
from oracle import block as ob

pytestmark = pytest.mark.gpu
ACT = {"none": 0, "silu": 1, "gelu": 2}


def _reverse(M, K, N, act, dtype, res, packed):
    """Runs both directions and checks the gradients. packed: whether W^T has to be laid out for the reverse pass."""
    import torch
    from paper_2506_21788_amd import binding as B
    print("dense reverse", M, K, N, act, dtype, res, flush=True)
    rng = np.random.default_rng(M + 3 * K + 7 * N)
    code = B.BF16 if dtype == "bf16" else B.F32
    x, W = rounded(rng.standard_normal((M, K)), dtype), rounded(rng.standard_normal((K, N)) * K ** -0.5, dtype)
    b, g = rounded(rng.standard_normal(N), "f32"), rounded(rng.standard_normal((M, N)), dtype)
    rx = rounded(rng.standard_normal((M, K)), dtype) if res else None
    ws_b, saved_b = B.dense_workspace_bytes(M, K, N, ACT[act], code)
    dact = 0 if act == "none" else (M * N * 4 + 255) // 256 * 256
    assert (saved_b > dact) == packed, "not the kernel that this case is for"
    (ws, wg), (saved, sg) = room(ws_b), room(saved_b)
    y, g_x, gW, g_b = empty((M, N), dtype), empty((M, K), dtype), empty((K, N)), empty(N)
    dx, dW, dg = dev(x, dtype), dev(W, dtype), dev(g, dtype)
    B.dense_fwd(M, K, N, ACT[act], code, dx, dW, dev(b), None, y, saved, ws)
    B.dense_bwd(M, K, N, ACT[act], code, dx, dW, saved, dg, g_x, gW, g_b, ws, r_x=dev(rx, dtype))
    torch.cuda.synchronize()
    assert untouched(wg, sg)
    # z off by (K + 8) half-steps of float32 of its sum of magnitudes; act' by 0.8 of that (its slope) and 16 half-steps of its own
    z, zm = x @ W + b, np.abs(x) @ np.abs(W) + np.abs(b)
    _, d = ob.activation(z, act)
    w_gx, w_gW, w_gb = ob.dense_bwd(x, W, b, act, g)
    gz = np.abs(g * d)
    egz = np.abs(g) * (0.8 * (K + 8) * U32 * zm + 16 * U32 * (1.0 + np.abs(z))) if act != "none" else np.zeros_like(gz)
    # bf16: g_z enters both products as two terms, the second the rounded remainder of the first: 2^-8 twice, 2^-16 of it is lost at most
    two = 2.0 ** -16 * gz if dtype == "bf16" and act != "none" else 0.0
    e = ((N + 8) * U32 * gz + egz + two) @ np.abs(W).T
    want = w_gx + (0.0 if rx is None else rx)
    close("g_x", g_x, want, e / U32 + np.abs(want), 1, dtype)
    e = np.abs(x).T @ ((M + 8) * U32 * gz + egz + two)
    close("gW", gW, w_gW, e / U32, 1)
    close("g_b", g_b, w_gb, (((M + 8) * U32 * gz + egz).sum(0)) / U32, 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,res", [("none", False), ("silu", True), ("gelu", False), ("none", True)])
@pytest.mark.parametrize("M,K,N,packed", [(4200, 1030, 70, True), (16500, 200, 131, True), (1000, 650, 45, False), (33, 70, 35, False), (8100, 513, 301, True)])
def test_g_x_keeps_g_z(M, K, N, packed, act, res, dtype):
    _reverse(M, K, N, act, dtype, res, packed)
