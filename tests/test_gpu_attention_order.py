"""Attention where a workgroup takes several tiles, where heads lie far apart and where sums are taken in turns; the terms of its weights (needs a GPU)."""
import numpy as np
import pytest

from block_util import U32, dev, empty
from oracle import block as ob
from test_gpu_attention import _check, _problem, _run

pytestmark = pytest.mark.gpu


def _common(P, rare, seed=0):
    """Most pairs into the last bucket, as in a large structure; the first rows keep a mixture."""
    rng = np.random.default_rng(seed)
    where, pitch = ob.pair_layout(P["off"])
    for k in range(P["G"]):
        n = int(P["off"][k + 1] - P["off"][k])
        m = P["pairs"][where[k]:where[k + 1]].reshape(n, pitch[k])
        common = (rng.random((n, n)) > rare) & (m[:, :n] < P["nb"])
        common[:40] = False
        m[:, :n][common] = P["nb"] - 1
    return P


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_graphs_with_more_tiles_than_workgroups(dtype):
    """64 heads have 64 workgroups each in the pass over queries, for 106 tiles: tables, sums and joins go on from tile to tile."""
    _check(_common(_problem([1100, 1029, 1100], 64, 8, 8, 6, dtype, left_out=0.02), 0.01))


@pytest.mark.parametrize("dtype,heads,kv,d", [("f32", 4, 2, 128), ("f32", 8, 4, 64), ("bf16", 4, 4, 128)])
@pytest.mark.parametrize("n", [1000, 1100])
def test_heads_far_apart(n, dtype, heads, kv, d):
    """Keys and values of a graph past 1 MB: its heads are dealt to different parts of the chip."""
    assert 2 * n * kv * d * (2 if dtype == "bf16" else 4) > 2e6
    P = _problem([n], heads, kv, d, 12, dtype, left_out=0.02)
    _check(_common(P, 0.01) if n > 1024 else P)


@pytest.mark.parametrize("drop_far", [False, True])
def test_sums_in_turn_repeat_themselves(drop_far):
    """Two pairs of one row that add to one word of LDS (16 keys apart, in one bucket): the same bits every time, and the right sum. drop_far:
    what is beyond the last boundary takes no part."""
    P = _problem([1090], 2, 1, 32, 9, "bf16", holes=False)
    m = P["pairs"][:1090 * 1120].reshape(1090, 1120)
    m[:, :1090] = 255 if drop_far else 8
    i = np.arange(1090)
    for step in (0, 16, 5):                     # in every row three near pairs, two of them a half tile apart
        m[i, (i + step) % 1090] = 3
    got = _check(P)
    for _ in range(3):
        assert all(np.array_equal(a, b) for a, b in zip(_run(P), got))


def test_weights_of_the_output_enter_whole():
    """All values of a graph are 1 and all of g_out too: dP = D = d exactly if the weights in the output are those of the row's sum, and then
    g_bias = 0. With two bf16 terms of each weight the output falls short of 1 by some 2^-17 and g_bias shows it."""
    n, G, d, nb = 5, 60, 8, 12
    P = _problem([n] * G, 1, 1, d, nb, "bf16", holes=False)
    P["qkv"][:, :2], P["qkv"][:, 2], P["g"][:] = 0.0, 1.0, 1.0
    got = _run(P)
    allowed, short = np.zeros(nb), np.zeros(nb)
    where, pitch = ob.pair_layout(P["off"])
    for k in range(G):
        m = P["pairs"][where[k]:where[k + 1]].reshape(n, pitch[k])[:, :n].astype(int)
        s = P["bias"][0][m]
        w = np.exp(s - s.max(1, keepdims=True)).astype(np.float32)
        p = w.astype(np.float64) / w.astype(np.float64).sum(1, keepdims=True)
        cut = lambda x: (x.view(np.uint32) & 0xffff0000).view(np.float32)  # noqa: E731
        two = cut(w) + cut(w - cut(w))
        delta = 1.0 - two.astype(np.float64).sum(1, keepdims=True) / w.astype(np.float64).sum(1, keepdims=True)
        # the products of n weights in three terms, their sum, the quotient, D's sum over d equal terms
        allowed += np.bincount(m.ravel(), weights=(p * d * (4 * n + 8) * U32).ravel(), minlength=nb)
        short += np.bincount(m.ravel(), weights=(p * d * delta).ravel(), minlength=nb)
    assert (short > 1.5 * allowed).all(), "a weight of two terms would not show"
    assert (np.abs(got[2][0]) <= allowed).all(), np.abs(got[2][0] / allowed).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_where_a_workgroup_takes_more_than_64_kb(dtype):
    import torch
    from paper_2506_21788_amd import binding as B
    P = _problem([400], 4, 1, 128, 64, dtype)
    N, code = P["N"], B.BF16 if dtype == "bf16" else B.F32
    args = (N, 1, 4, 1, 128, 64, code, P["scale"])
    plan = torch.empty(B.pair_plan_workspace_bytes(N, 1), dtype=torch.uint8, device="cuda")
    B.pair_plan(N, 1, dev(P["off"], "i32"), plan)
    ws_b, saved_b = B.graph_attention_workspace_bytes(*args[:7])
    ws, saved = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    pairs, qkv, bias, g = dev(P["pairs"], "u8"), dev(P["qkv"], dtype), dev(P["bias"]), dev(P["g"], dtype)
    res = [empty((N, 4, 128), dtype), empty((N, 6, 128), dtype), empty((4, 64))]

    def both():
        B.graph_attention_fwd(*args, plan, pairs, qkv, bias, res[0], saved)
        B.graph_attention_bwd(*args, plan, pairs, qkv, bias, res[0], saved, g, res[1], res[2], ws)

    both()
    torch.cuda.synchronize()
    want = [r.clone() for r in res]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for r in res:
            r.fill_(float("nan"))
        ws.fill_(255)
        saved.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(res, want))
        both()
        torch.cuda.synchronize()


def test_long_sums_of_the_bias_gradient():
    """All pairs of the last bucket have one and the same ds, c, of 24 bits: a lane that added its 2,048 one after the other would be off by
    the same rounding again and again. One key of 16,384 has a value, v; equal weights: p = 2^-14, D = v / 16384, c = -v 2^-28, all exact."""
    import torch
    from paper_2506_21788_amd import binding as B
    n, d, nb, v = 16384, 8, 3, np.float32(1.5555555)
    c = np.float32(v * np.float32(2.0 ** -28))
    one = np.float32(0.0)
    for _ in range(2048):
        one = np.float32(one + c)
    # a tile's sixteen, 128 tiles of a wavefront, the other half, 32 columns in eight chains, four wavefronts, the result's own rounding
    allowed = (16 + 128 + 2 + 4 + 3 + 4 + 1) * U32
    assert abs(float(one) / (2048 * float(c)) - 1.0) > 1.5 * allowed, "a chain of 2,048 would not show"
    plan = torch.empty(B.pair_plan_workspace_bytes(n, 1), dtype=torch.uint8, device="cuda")
    size = B.pair_plan(n, 1, dev(np.array([0, n]), "i32"), plan)
    pairs = torch.full((size,), 2, dtype=torch.uint8, device="cuda")
    pairs.view(n, n)[:, 0] = 0
    qkv, g, bias = torch.zeros((n, 3, d), device="cuda"), torch.zeros((n, 1, d), device="cuda"), torch.zeros((1, nb), device="cuda")
    qkv[0, 2, 0], g[:, 0, 0] = float(v), 1.0
    ws_b, saved_b = B.graph_attention_workspace_bytes(n, 1, 1, 1, d, nb, B.F32)
    ws, saved = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    out, g_qkv, g_bias = torch.empty_like(g), torch.empty_like(qkv), torch.empty_like(bias)
    B.graph_attention_fwd(n, 1, 1, 1, d, nb, B.F32, 1.0, plan, pairs, qkv, bias, out, saved)
    B.graph_attention_bwd(n, 1, 1, 1, d, nb, B.F32, 1.0, plan, pairs, qkv, bias, out, saved, g, g_qkv, g_bias, ws)
    got = g_bias.double().cpu().numpy()[0]
    assert (out[:, 0, 0] == float(v) / n).all()
    want = np.array([n * 2.0 ** -14 * (float(v) - float(v) / n), 0.0, -n * (n - 1) * float(c)])
    assert (np.abs(got - want) <= allowed * np.abs(want)).all(), np.abs(got / np.where(want == 0, 1, want) - 1) / allowed


def test_bias_gradient_has_no_drift():
    """The sum of g_bias for g_out and for -g_out: every rounding to nearest is the same for both but for its sign, so what is left is a drift of
    the matrix cores' sums, which are low by some 6e-10 for 32 terms of size 1, whatever their sign. Rows must not add it up."""
    import torch
    from paper_2506_21788_amd import binding as B
    n, d = 4096, 32
    gen = torch.Generator(device="cuda").manual_seed(5)
    plan = torch.empty(B.pair_plan_workspace_bytes(n, 1), dtype=torch.uint8, device="cuda")
    pairs = torch.zeros(B.pair_plan(n, 1, dev(np.array([0, n]), "i32"), plan), dtype=torch.uint8, device="cuda")
    qkv = torch.zeros((n, 3, d), dtype=torch.bfloat16, device="cuda")
    qkv[:, 2] = torch.randn((n, d), device="cuda", generator=gen).to(torch.bfloat16)
    g = torch.randn((n, 1, d), device="cuda", generator=gen).to(torch.bfloat16)
    bias = torch.zeros((1, 1), device="cuda")
    ws_b, saved_b = B.graph_attention_workspace_bytes(n, 1, 1, 1, d, 1, B.BF16)
    ws, saved = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    out, g_qkv, both = torch.empty_like(g), torch.empty_like(qkv), [torch.empty_like(bias), torch.empty_like(bias)]
    B.graph_attention_fwd(n, 1, 1, 1, d, 1, B.BF16, 1.0, plan, pairs, qkv, bias, out, saved)
    for sign, res in zip((1.0, -1.0), both):
        B.graph_attention_bwd(n, 1, 1, 1, d, 1, B.BF16, 1.0, plan, pairs, qkv, bias, out, saved, g * sign, g_qkv, res, ws)
    drift = float(both[0].double() + both[1].double()) / (2 * n)
    # a sixth of what one sum is low by; half a step of the two results, of size 1e-4 at most, is 1e-15 a row
    assert abs(drift) <= 1e-10, drift


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graphs_of_one_atom_have_no_gradient_but_the_rounding(dtype):
    """An atom that attends to itself alone: ds is what two float32 products of the same numbers differ by, and g_q and g_k no more than that."""
    _check(_problem([1] * 700, 8, 4, 8, 2, dtype, holes=False))
