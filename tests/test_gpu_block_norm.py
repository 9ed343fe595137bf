"""The seam of two blocks (norms, gate, residual scale) against float64, forward and reverse (needs a GPU)."""
import numpy as np
import pytest

from block_util import close, dev, empty, room, rounded, untouched
from oracle import block as ob

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _case(N, H, layer, gate, dtype, post=True, pre=True, g_res=True, seed=0, x_scale=2.0, offset=0.5):
    import torch
    from paper_2506_21788_amd import binding as B
    print("block_norm", N, H, layer, gate, dtype, post, pre, g_res, flush=True)
    rng = np.random.default_rng(seed + 131 * N + H)
    f32 = lambda a: rounded(a, "f32")  # noqa: E731
    x, P = f32(x_scale * rng.standard_normal((N, H)) + offset), f32(rng.standard_normal((5, H)))
    b = rounded(rng.standard_normal((N, H)), dtype) if post else None
    z = rounded(2 * rng.standard_normal((N, 1 if gate == "atom" else H)), dtype) if gate else None
    gx = f32(rng.standard_normal((N, H))) if g_res else None
    gy = rounded(rng.standard_normal((N, H)), dtype) if pre else None
    norm, gt = B.NORM_LAYER if layer else B.NORM_RMS, {None: B.GATE_NONE, "atom": B.GATE_ATOM, "channel": B.GATE_CHANNEL}[gate]
    dt = B.BF16 if dtype == "bf16" else B.F32

    ws_b, saved_b = B.block_norm_workspace_bytes(N, H)
    (ws, wg), (saved, sg) = room(ws_b), room(saved_b)
    d = dict(x=dev(x), b=dev(b, dtype), z=dev(z, dtype), P=dev(P))
    x_out, y = empty((N, H)) if post else None, empty((N, H), dtype) if pre else None
    B.block_norm_fwd(N, H, norm, gt, dt, EPS, d["x"], d["b"], d["z"], d["P"], x_out, y, saved)
    x1, y1 = ob.block_norm_fwd(x, b, z, P, layer, EPS, pre)

    # what the results are made of: the same sums over magnitudes
    s, w1, c1, w0, c0 = np.abs(P)

    def parts(u):
        mu = np.abs(u).mean(1, keepdims=True) if layer else 0.0
        _, r = ob.standardise(u, layer, EPS)
        return (np.abs(u) + mu) * r, r

    gamma = 1.0 if z is None else ob.sigmoid(z)
    m1 = np.abs(x)
    if post:
        bm, rb = parts(b)
        um = bm * w1 + c1
        m1 = m1 + s * gamma * um
    xm, rx = parts(x1)
    xm = xm + m1 * rx
    # a row's two sums in float32 (a tree: log2 H additions deep, some of them a lane's own), the root, the division, the products
    fwd = 16 + np.log2(H) + 16
    if post:
        close("x_out", x_out, x1, m1, fwd)
    if pre:
        close("y", y, y1, xm * w0 + c0 + np.abs(y1), 2 * fwd, dtype)

    g_x, gP = empty((N, H)), empty((5, H))
    g_b, g_z = (empty((N, H), dtype) if post else None), (empty(z.shape, dtype) if gate else None)
    B.block_norm_bwd(N, H, norm, gt, dt, x_out if post else d["x"], d["b"], d["z"], d["P"], saved, dev(gx), dev(gy, dtype), g_x,
                     g_b, g_z, gP, ws)
    torch.cuda.synchronize()
    assert untouched(wg, sg)
    want = ob.block_norm_bwd(x, b, z, P, layer, EPS, gx, gy)
    gm = np.zeros((N, H)) if gx is None else np.abs(gx)
    Pm = np.zeros((5, H))
    if pre:
        t = np.abs(gy) * w0
        Pm[3], Pm[4] = (np.abs(gy) * xm).sum(0), np.abs(gy).sum(0)
        gm = gm + rx * (t + (t.mean(1, keepdims=True) if layer else 0.0) + xm * (t * xm).mean(1, keepdims=True)) * (1 + xm)
    bwd = 4 * fwd
    close("g_x", g_x, want[0], gm, bwd)
    if post:
        q = gm * s * gamma
        Pm[0], Pm[1], Pm[2] = (gm * gamma * um).sum(0), (q * bm).sum(0), q.sum(0)
        t = q * w1
        close("g_b", g_b, want[1], rb * (t + (t.mean(1, keepdims=True) if layer else 0.0) + bm * (t * bm).mean(1, keepdims=True)) * (1 + bm),
              2 * bwd, dtype)
        if gate:
            zm = q * um
            close("g_z", g_z, want[2], zm.sum(1, keepdims=True) if gate == "atom" else zm, 2 * bwd, dtype)
    # sums over N rows: of a workgroup's rows one after the other, then over the workgroups
    close("gP", gP, want[3], Pm, 2 * bwd + N)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,H", [(1, 1), (3, 2), (5, 3), (2, 63), (17, 64), (9, 128), (33, 130), (11, 256), (7, 260), (13, 511), (6, 866),
                                 (4, 889), (5, 1000), (3, 1024), (2500, 64), (4200, 96)])
def test_sizes(N, H, dtype):
    for layer, gate in ((False, "channel"), (True, "atom")):
        _case(N, H, layer, gate, dtype)


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", [None, "atom", "channel"])
def test_every_form(layer, gate):
    for kw in (dict(), dict(pre=False), dict(g_res=False)):
        _case(37, 100, layer, gate, "bf16", **kw)
    if gate is None:
        _case(37, 100, layer, None, "f32", post=False)
        _case(37, 100, layer, None, "bf16", post=False, g_res=False)


def test_rows_of_zeros_and_constant_rows():
    import torch
    from paper_2506_21788_amd import binding as B
    H = 48
    x = torch.zeros((3, H), device="cuda")
    x[1], x[2] = 3.0, -1e18
    P = torch.ones((5, H), device="cuda")
    for norm in (B.NORM_RMS, B.NORM_LAYER):
        y = empty((3, H))
        B.block_norm_fwd(3, H, norm, B.GATE_NONE, B.F32, EPS, x, None, None, P, None, y, None)
        got = y.cpu()
        assert torch.equal(got[0], torch.ones(H))                       # nothing but the shift
        if norm == B.NORM_LAYER:
            assert torch.equal(got[1], torch.ones(H)) and torch.isfinite(got[2]).all()
        else:
            assert torch.allclose(got[1], torch.full((H,), 2.0), atol=1e-5) and torch.allclose(got[2], torch.zeros(H), atol=1e-5)


def test_in_place_gate_extremes_and_no_rows():
    import torch
    from paper_2506_21788_amd import binding as B
    N, H = 21, 72
    g = torch.Generator(device="cuda").manual_seed(3)
    x, b = (torch.randn((N, H), device="cuda", generator=g) for _ in range(2))
    z = torch.full((N, H), 200.0, device="cuda")
    z[::2] = -200.0                                                     # closed: nothing is added
    P = torch.randn((5, H), device="cuda", generator=g)
    out, same = empty((N, H)), x.clone()
    B.block_norm_fwd(N, H, B.NORM_RMS, B.GATE_CHANNEL, B.F32, EPS, x, b, z, P, out, None, None)
    B.block_norm_fwd(N, H, B.NORM_RMS, B.GATE_CHANNEL, B.F32, EPS, same, b, z, P, same, None, None)
    assert torch.equal(out, same) and torch.equal(out[::2], x[::2]) and not torch.equal(out[1::2], x[1::2])
    none = torch.empty((0, H), device="cuda")
    gP = empty((5, H))
    B.block_norm_fwd(0, H, B.NORM_RMS, B.GATE_NONE, B.F32, EPS, none, none, None, P, none, none, None)
    B.block_norm_bwd(0, H, B.NORM_RMS, B.GATE_NONE, B.F32, none, none, None, P, None, none, none, none, none, None, gP, None)
    assert torch.equal(gP, torch.zeros_like(gP))


def test_reverse_pass_in_a_graph_on_another_stream():
    import torch
    from paper_2506_21788_amd import binding as B
    N, H = 3000, 256
    g = torch.Generator(device="cuda").manual_seed(4)
    x, b, z, gx, gy = (torch.randn((N, H), device="cuda", generator=g) for _ in range(5))
    P = torch.randn((5, H), device="cuda", generator=g)
    ws_b, saved_b = B.block_norm_workspace_bytes(N, H)
    ws, saved = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    out = [torch.empty((N, H), device="cuda") for _ in range(5)] + [torch.empty((5, H), device="cuda")]

    def both():
        B.block_norm_fwd(N, H, B.NORM_LAYER, B.GATE_CHANNEL, B.F32, EPS, x, b, z, P, out[0], out[1], saved)
        B.block_norm_bwd(N, H, B.NORM_LAYER, B.GATE_CHANNEL, B.F32, out[0], b, z, P, saved, gx, gy, out[2], out[3], out[4], out[5], ws)

    both()
    torch.cuda.synchronize()
    want = [o.clone() for o in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for o in out:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(out, want))
