"""Dense products with bias, activation and residual against float64, forward and reverse (needs a GPU)."""
import numpy as np
import pytest

from block_util import U32, UBF, close, dev, empty, room, rounded, untouched
from oracle import block as ob

pytestmark = pytest.mark.gpu
ACT = {"none": 0, "silu": 1, "gelu": 2}


def _case(M, K, N, act, dtype, bias=True, res=False, want_gx=True, seed=0, scale=1.0):
    import torch
    from paper_2506_21788_amd import binding as B
    print("dense", M, K, N, act, dtype, bias, res, flush=True)
    rng = np.random.default_rng(seed + M + 3 * K + 7 * N)
    bf, code = dtype == "bf16", B.BF16 if dtype == "bf16" else B.F32
    x, W = rounded(scale * rng.standard_normal((M, K)), dtype), rounded(rng.standard_normal((K, N)) * K ** -0.5, dtype)
    b = rounded(rng.standard_normal(N), "f32") if bias else None
    r = rounded(rng.standard_normal((M, N)), dtype) if res else None
    g = rounded(rng.standard_normal((M, N)), dtype)
    ws_b, saved_b = B.dense_workspace_bytes(M, K, N, ACT[act], code)
    (ws, wg), (saved, sg) = room(ws_b), room(saved_b)
    dx, dW, db, dg = dev(x, dtype), dev(W, dtype), dev(b), dev(g, dtype)
    y, alone, g_x = empty((M, N), dtype), empty((M, N), dtype), empty((M, K), dtype) if want_gx else None
    gW, g_b = empty((K, N)), empty(N) if bias else None
    B.dense_fwd(M, K, N, ACT[act], code, dx, dW, db, dev(r, dtype), y, saved, ws)
    B.dense_fwd(M, K, N, ACT[act], code, dx, dW, db, dev(r, dtype), alone, None, ws)
    rx = rounded(rng.standard_normal((M, K)), dtype) if want_gx and res else None
    B.dense_bwd(M, K, N, ACT[act], code, dx, dW, saved, dg, g_x, gW, g_b, ws, r_x=dev(rx, dtype))
    torch.cuda.synchronize()
    assert untouched(wg, sg) and torch.equal(y.view(torch.uint8), alone.view(torch.uint8))

    # z is off by K half-steps of float32 of the sum of magnitudes (6 more for the terms of a split operand); an activation's slope is at
    # most 1.13 and its curvature at most 0.8, and it adds 16 half-steps of its own
    z = x @ W + (0.0 if b is None else b)
    zm = np.abs(x) @ np.abs(W) + (0.0 if b is None else np.abs(b))
    ez = (K + 8) * U32 * zm
    a, d = ob.activation(z, act)
    want = a + (0.0 if r is None else r)
    close("y", y, want, (1.13 * ez / U32 + 16 * (np.abs(a) + np.abs(z) * 0.01) + np.abs(want)) if act != "none" else ez / U32 + np.abs(want), 1, dtype)
    w_gx, w_gW, w_gb = ob.dense_bwd(x, W, b, act, g)
    gz = np.abs(g * d)
    egz = np.abs(g) * (0.8 * ez + 16 * U32 * (1.0 + np.abs(z))) if act != "none" else np.zeros_like(gz)
    if want_gx:
        e = ((N + 8) * U32 * gz + egz + (UBF * gz if bf and act != "none" else 0.0)) @ np.abs(W).T
        rx = 0.0 if rx is None else rx
        close("g_x", g_x, w_gx + rx, e / U32 + np.abs(w_gx + rx), 1, dtype)
    # bf16: g_z enters gW as two terms, UBF^2 of it is lost
    e = np.abs(x).T @ ((M + 8) * U32 * gz + egz + (UBF ** 2 * gz if bf and act != "none" else 0.0))
    close("gW", gW, w_gW, e / U32, 1)
    if bias:
        close("g_b", g_b, w_gb, (((M + 8) * U32 * gz + egz).sum(0)) / U32, 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 17, 3), (3, 64, 65), (33, 31, 32), (65, 128, 130), (187, 128, 384), (700, 64, 200),
                                   (2100, 130, 96), (5000, 257, 129)])
def test_sizes(M, K, N, act, dtype):
    _case(M, K, N, act, dtype, res=(M + K) % 2 == 0, bias=N != 65)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_tiles_with_odd_edges(dtype):
    _case(9001, 300, 515, "silu", dtype, res=True)
    _case(8200, 889, 866, "none", dtype, want_gx=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_column_and_one_long_contraction(dtype):
    _case(3000, 4100, 1, "gelu", dtype)
    _case(40, 1, 2050, "silu", dtype)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_far_arguments_of_the_activations(act):
    import torch
    from paper_2506_21788_amd import binding as B
    z = torch.tensor([[-1e4, -200.0, -90.0, -20.0, -1e-30, 0.0, 1e-30, 20.0, 90.0, 200.0, 1e4]], device="cuda")
    n = z.shape[1]
    one = torch.eye(n, device="cuda")
    ws_b, saved_b = B.dense_workspace_bytes(1, n, n, ACT[act], B.F32)
    saved, y, g_x, gW = torch.empty(saved_b, dtype=torch.uint8, device="cuda"), empty((1, n)), empty((1, n)), empty((n, n))
    B.dense_fwd(1, n, n, ACT[act], B.F32, z, one, None, None, y, saved, None)
    B.dense_bwd(1, n, n, ACT[act], B.F32, z, one, saved, torch.ones((1, n), device="cuda"), g_x, gW, None, torch.empty(max(ws_b, 16), dtype=torch.uint8, device="cuda"))
    a, d = ob.activation(z.double().cpu().numpy(), act)
    assert np.allclose(y.cpu().numpy(), a, rtol=1e-5, atol=1e-7) and np.allclose(g_x.cpu().numpy(), d, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows_and_in_place_residual(dtype):
    import torch
    from paper_2506_21788_amd import binding as B
    code = B.BF16 if dtype == "bf16" else B.F32
    gW, g_b, none = empty((5, 7)), empty(7), empty((0, 5), dtype)
    B.dense_fwd(0, 5, 7, 1, code, none, none, None, None, none, None, None)
    B.dense_bwd(0, 5, 7, 1, code, none, none, None, none, none, gW, g_b, None)
    assert torch.equal(gW, torch.zeros_like(gW)) and torch.equal(g_b, torch.zeros_like(g_b))
    x, W, r = (dev(np.random.default_rng(k).standard_normal((70, 70)), dtype) for k in range(3))
    y = empty((70, 70), dtype)
    B.dense_fwd(70, 70, 70, 1, code, x, W, None, r, y, None, None)
    B.dense_fwd(70, 70, 70, 1, code, x, W, None, r, r, None, None)
    assert torch.equal(y, r)


@pytest.mark.parametrize("n", [0, 1, 7, 8, 9, 2049, 100003])
def test_round_bf16(n):
    import torch
    from paper_2506_21788_amd import binding as B
    x = torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    if n > 4:
        x[:4] = torch.tensor([float("nan"), float("inf"), 1.00390625, 3.4e38])     # 1 + 2^-8: a tie
    out = torch.full((n + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    B.round_bf16(x, out[:n])
    want = x.to(torch.bfloat16)
    assert torch.equal(torch.nan_to_num(out[:n]), torch.nan_to_num(want)) and bool((out[n:] == 7.0).all())


def test_in_a_graph_on_another_stream():
    import torch
    from paper_2506_21788_amd import binding as B
    M, K, N = 4000, 200, 300
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, W, g = (torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16) for s in ((M, K), (K, N), (M, N)))
    b = torch.randn(N, device="cuda", generator=gen)
    ws_b, saved_b = B.dense_workspace_bytes(M, K, N, 1, B.BF16)
    ws, saved = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    out = [empty((M, N), "bf16"), empty((M, K), "bf16"), empty((K, N)), empty(N)]

    def both():
        B.dense_fwd(M, K, N, 1, B.BF16, x, W, b, None, out[0], saved, ws)
        B.dense_bwd(M, K, N, 1, B.BF16, x, W, saved, g, out[1], out[2], out[3], ws)

    both()
    torch.cuda.synchronize()
    want = [o.clone() for o in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for o in out:
            o.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(out, want))
