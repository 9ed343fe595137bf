"""Attention over the atoms of each graph with a learned bias per bucket, forward and reverse, against float64 (needs a GPU)."""
import numpy as np
import pytest

from block_util import U32, UBF, dev, empty, room, rounded, untouched
from oracle import block as ob

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -126


def _problem(sizes, heads, kv, d, nb, dtype, left_out=0.1, seed=0, holes=True):
    rng = np.random.default_rng(seed + sum(sizes) + 7 * d + heads)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    N = int(off[-1])
    qkv, g = rounded(rng.standard_normal((N, heads + 2 * kv, d)), dtype), rounded(rng.standard_normal((N, heads, d)), dtype)
    bias = rounded(rng.standard_normal((heads, nb)), "f32")
    where, pitch = ob.pair_layout(off)
    pairs = rng.integers(0, 256, where[-1]).astype(np.uint8)       # padding: anything
    absent = np.zeros(N, bool)
    for k, (a, e) in enumerate(zip(off[:-1], off[1:])):
        n = int(e - a)
        m = rng.integers(0, nb, (n, n))
        if holes:
            m = np.where(rng.random((n, n)) < left_out, rng.integers(nb, 256, (n, n)), m)
            out = rng.random(n) < left_out
            m[out] = ob.PAIR_NONE                                  # atoms that are nobody's partner: an empty row and an empty column
            m[:, out] = ob.PAIR_NONE
            absent[a:e] = out
        pairs[where[k]:where[k + 1]].reshape(n, pitch[k])[:, :n] = m
    return dict(off=off, N=N, G=len(sizes), heads=heads, kv=kv, d=d, nb=nb, dtype=dtype, qkv=qkv, g=g, bias=bias, pairs=pairs,
                scale=d ** -0.5, absent=absent)


def _allowed(P, out, g_qkv, g_bias):
    """How far the results may be off: rounding errors carried through the formulas, in absolute values.

    A dot product of d terms is off by (d + 4) half-steps of its sum of magnitudes, the exponent by that and its own rounding,
    so a weight by er relative; sums of n terms add n half-steps. bf16 adds a half-step of bf16 where an operand is rounded
    (ds and p in the reverse products; its square for the output's weights, which enter as two terms). A weight below 2^-126, the
    smallest normal number of float32, may come out as zero: TINY absolute."""
    off, heads, kv, d, nb = P["off"], P["heads"], P["kv"], P["d"], P["nb"]
    bf, rep, scale = P["dtype"] == "bf16", P["heads"] // P["kv"], P["scale"]
    qkv, bias, g = np.nan_to_num(P["qkv"], posinf=0.0, neginf=0.0), P["bias"], np.nan_to_num(P["g"], posinf=0.0, neginf=0.0)
    where, pitch = ob.pair_layout(off)
    t_out, t_qkv, t_bias = np.zeros(out.shape), np.zeros(qkv.shape), np.zeros(g_bias.shape)
    count = 0
    for k, (a, e) in enumerate(zip(off[:-1], off[1:])):
        n = int(e - a)
        if n == 0:
            continue
        m = P["pairs"][where[k]:where[k + 1]].reshape(n, pitch[k])[:, :n].astype(np.int64)
        live = m < nb
        mc = np.where(live, m, 0)
        count += n * n
        for h in range(heads):
            q, kk, v = qkv[a:e, h], qkv[a:e, heads + h // rep], qkv[a:e, heads + kv + h // rep]
            b = bias[h][mc]
            s = scale * q @ kk.T + b
            fin = np.where(np.isfinite(b), np.abs(b), 0.0)
            es = U32 * ((d + 4) * scale * np.abs(q) @ np.abs(kk).T + 4 * fin + 4 * np.where(np.isfinite(s), np.abs(s), 0.0))
            ok = live & (b > -np.inf)
            top = np.where(ok, s, -np.inf).max(1, keepdims=True)
            ex = np.where(ok, np.exp(np.where(ok, s, 0.0) - np.where(np.isfinite(top), top, 0.0)), 0.0)
            tot = ex.sum(1, keepdims=True)
            p = ex / np.where(tot == 0, 1.0, tot)
            er = es + np.where(ok, es, 0.0).max(1, keepdims=True) + (n + 16) * U32
            o, go = out[a:e, h], g[a:e, h]
            eo = (p * (er + (n + 8) * U32 + (UBF ** 2 if bf else 0.0)) + TINY * ok) @ np.abs(v)
            t_out[a:e, h] = eo + (UBF * (np.abs(o) + eo) if bf else 0.0)
            dp, edp = np.abs(go @ v.T), (d + 4) * U32 * np.abs(go) @ np.abs(v).T
            D, eD = np.abs((go * o).sum(1))[:, None], ((np.abs(go) * eo).sum(1) + (d + 4) * U32 * (np.abs(go) * np.abs(o)).sum(1))[:, None]
            ds = p * (dp + D)
            eds = p * ((er + 4 * U32) * (dp + D) + edp + eD) + TINY * ok * (dp + D)
            w = eds + (UBF if bf else 0.0) * ds + (n * rep + 8) * U32 * ds
            t_qkv[a:e, h] += scale * w @ np.abs(kk)
            t_qkv[a:e, heads + h // rep] += scale * w.T @ np.abs(q)
            t_qkv[a:e, heads + kv + h // rep] += (p * (er + (UBF if bf else 0.0) + (n * rep + 8) * U32) + TINY * ok).T @ np.abs(go)
            # a bucket's sum: a lane's pairs one after the other, then 64 lanes, then the wavefronts
            t_bias[h] += np.bincount(mc[ok], weights=(eds + (n + 512) * U32 * ds)[ok], minlength=nb)[:nb]
    if bf:
        t_qkv += UBF * (np.abs(g_qkv) + t_qkv)
    return t_out, t_qkv, t_bias


def _run(P, keep=True):
    import torch
    from paper_2506_21788_amd import binding as B
    N, G, h, kv, d, nb, dt = P["N"], P["G"], P["heads"], P["kv"], P["d"], P["nb"], P["dtype"]
    print("graph_attention", N, G, h, kv, d, nb, dt, flush=True)
    code = B.BF16 if dt == "bf16" else B.F32
    plan = torch.empty(B.pair_plan_workspace_bytes(N, G), dtype=torch.uint8, device="cuda")
    size = B.pair_plan(N, G, dev(P["off"], "i32"), plan)
    assert size == P["pairs"].size
    ws_b, saved_b = B.graph_attention_workspace_bytes(N, G, h, kv, d, nb, code)
    (ws, wg), (saved, sg) = room(ws_b), room(saved_b)
    pairs, qkv, bias, g = dev(P["pairs"], "u8"), dev(P["qkv"], dt), dev(P["bias"]), dev(P["g"], dt)
    out, alone, g_qkv, g_bias = empty((N, h, d), dt), empty((N, h, d), dt), empty((N, h + 2 * kv, d), dt), empty((h, nb))
    B.graph_attention_fwd(N, G, h, kv, d, nb, code, P["scale"], plan, pairs, qkv, bias, out, saved)
    B.graph_attention_fwd(N, G, h, kv, d, nb, code, P["scale"], plan, pairs, qkv, bias, alone, None)
    B.graph_attention_bwd(N, G, h, kv, d, nb, code, P["scale"], plan, pairs, qkv, bias, out, saved, g, g_qkv, g_bias, ws)
    torch.cuda.synchronize()
    assert untouched(wg, sg)
    assert torch.equal(out.view(torch.uint8), alone.view(torch.uint8))
    return [t.double().cpu().numpy() for t in (out, g_qkv, g_bias)]


def _check(P):
    got = _run(P)
    want = ob.graph_attention(P["qkv"], P["bias"], P["pairs"], P["off"], P["heads"], P["kv"], P["scale"], P["g"])
    for name, a, w, t in zip(("out", "g_qkv", "g_bias"), got, want, _allowed(P, *want)):
        assert np.isfinite(a).all(), name
        over = np.abs(a - w) / (t + 1e-37)
        assert over.max(initial=0.0) <= 1.0, f"{name}: {over.max():.3g} of what is allowed at {np.unravel_index(over.argmax(), over.shape)}"
    return got


BATCHES = {"one atom": [1], "odd ends": [0, 13, 0, 1, 2, 0], "tile edges": [31, 32, 33, 63, 64, 65], "molecules": [5, 60, 17, 44, 9, 38],
           "crystals": [100, 200, 7, 161], "long": [523]}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("heads,kv,d,nb", [(1, 1, 8, 1), (4, 2, 32, 32), (3, 1, 40, 7), (2, 2, 64, 64), (4, 1, 128, 64)])
def test_batches(batch, heads, kv, d, nb, dtype):
    _check(_problem(BATCHES[batch], heads, kv, d, nb, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_pair_left_out(dtype):
    _check(_problem([90, 3, 33], 2, 2, 16, 5, dtype, holes=False))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,d,nb,rare", [(2, 1, 32, 16, 0.01), (1, 1, 64, 64, 0.02), (2, 2, 8, 2, 0.002), (1, 1, 128, 5, 1.0), (1, 1, 16, 1, 1.0)])
def test_long_graphs(heads, kv, d, nb, rare, dtype):
    """Over 1,024 atoms: most tiles have nearly all pairs in the last bucket, some have not (the first rows), some pairs are left out."""
    P = _problem([1100, 1029], heads, kv, d, nb, dtype, left_out=0.02)
    rng = np.random.default_rng(nb)
    where, pitch = ob.pair_layout(P["off"])
    for k, n in enumerate((1100, 1029)):
        m = P["pairs"][where[k]:where[k + 1]].reshape(n, pitch[k])
        common = (rng.random((n, n)) > rare) & (m[:, :n] < nb)
        common[:40] = False
        m[:, :n][common] = nb - 1
    _check(P)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_tiles_than_wavefronts(dtype):
    """Many heads: a wavefront takes several tiles, and its sums of the bias gradient run over them."""
    _check(_problem([1 + (5 * i) % 41 for i in range(150)], 64, 16, 8, 9, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[40, 70, 9], [300]])
def test_what_is_left_out_may_hold_anything(dtype, sizes):
    P = _problem(sizes, 4, 2, 24, 6, dtype, left_out=0.2)
    _check(P)
    P["qkv"], P["g"] = P["qkv"].copy(), P["g"].copy()
    junk = np.array([np.nan, np.inf, -np.inf])
    who = np.nonzero(P["absent"])[0]
    P["qkv"][who] = junk[np.arange(len(who)) % 3][:, None, None]
    P["g"][who] = junk[(np.arange(len(who)) + 1) % 3][:, None, None]
    got = _check(P)     # (not bit for bit as before: tiles that such values reach are formed in another order)
    assert len(who) > 3
    for a in got[:2]:
        assert (a[who] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_numbers_that_are_none_stay_where_they_count(dtype):
    """A NaN in one key: its graph's rows that attend to it are NaN, all others are as without it."""
    P = _problem([50, 60], 2, 1, 16, 4, dtype)
    clean = _run(P)
    j = int(np.nonzero(~P["absent"][:50])[0][3])
    P["qkv"] = P["qkv"].copy()
    P["qkv"][j, 2, 5] = np.nan
    got = _run(P)
    m = P["pairs"][:50 * 64].reshape(50, 64)[:, :50]
    hit = np.zeros(110, bool)
    hit[:50] = m[:, j] < 4
    assert 0 < hit.sum() < 50 and np.isnan(got[0][hit]).all()
    assert np.allclose(got[0][~hit], clean[0][~hit], rtol=2e-2 if dtype == "bf16" else 1e-5, atol=1e-6)
    assert np.array_equal(got[0][50:], clean[0][50:]) and np.array_equal(got[1][50:], clean[1][50:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_biases_of_the_lowest_value_and_of_minus_infinity(dtype):
    P = _problem([37, 70], 2, 2, 16, 3, dtype)
    low = float(np.finfo(np.float32).min)
    P["bias"] = np.array([[low, low, low], [0.5, -np.inf, low]])
    got = _run(P)
    off, (where, pitch) = P["off"], ob.pair_layout(P["off"])
    for k, (a, e) in enumerate(zip(off[:-1], off[1:])):
        n = e - a
        m = P["pairs"][where[k]:where[k + 1]].reshape(n, pitch[k])[:, :n]
        v = P["qkv"][a:e, 4]
        for i in range(n):
            live = m[i] < 3
            want = v[live].mean(0) if live.any() else np.zeros(16)     # all at the lowest value: equal weights
            assert np.allclose(got[0][a + i, 0], want, atol=1e-2 if dtype == "bf16" else 1e-5)
    P["bias"][0] = 0.0
    P["bias"][1] = [0.5, -np.inf, -1.0]
    _check(P)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("far", [-1e9, float(np.finfo(np.float32).min)])
def test_gradients_of_rows_of_far_biases(far, dtype):
    """Every bias of a head at one far value: at that size float32 holds no score, the weights are equal, forward and reverse."""
    P = _problem([45, 80], 2, 1, 16, 1, dtype, holes=False)
    P["bias"] = np.full((2, 1), far)
    P["qkv"] = np.concatenate([np.zeros_like(P["qkv"][:, :2]), P["qkv"][:, 2:]], 1)      # scores of zero: exactly the same weights
    got = _run(P)
    P["bias"] = np.zeros((2, 1))
    want = ob.graph_attention(P["qkv"], P["bias"], P["pairs"], P["off"], 2, 1, P["scale"], P["g"])
    for a, w, t in zip(got, want, _allowed(P, *want)):
        assert (np.abs(a - w) <= t + 1e-37).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(dtype):
    """Scores of some hundred: one weight of a row is nearly 1, the others vanish."""
    P = _problem([64, 100], 2, 2, 32, 4, dtype)
    P["qkv"] = rounded(P["qkv"] * 12.0, dtype)
    _check(P)


@pytest.mark.parametrize("sizes", [[60, 7, 130], [400]])
def test_in_a_graph_on_another_stream(sizes):
    import torch
    from paper_2506_21788_amd import binding as B
    P = _problem(sizes, 4, 2, 32, 8, "bf16")
    N, G = P["N"], P["G"]
    args = (N, G, 4, 2, 32, 8, B.BF16, P["scale"])
    plan = torch.empty(B.pair_plan_workspace_bytes(N, G), dtype=torch.uint8, device="cuda")
    B.pair_plan(N, G, dev(P["off"], "i32"), plan)
    ws_b, saved_b = B.graph_attention_workspace_bytes(*args[:6], B.BF16)
    ws, saved = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    pairs, qkv, bias, g = dev(P["pairs"], "u8"), dev(P["qkv"], "bf16"), dev(P["bias"]), dev(P["g"], "bf16")
    out, g_qkv, g_bias = empty((N, 4, 32), "bf16"), empty((N, 8, 32), "bf16"), empty((4, 8))

    def both():
        B.graph_attention_fwd(*args, plan, pairs, qkv, bias, out, saved)
        B.graph_attention_bwd(*args, plan, pairs, qkv, bias, out, saved, g, g_qkv, g_bias, ws)

    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, g_qkv, g_bias)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in (out, g_qkv, g_bias):
            t.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip((out, g_qkv, g_bias), want))


def test_offsets_past_32_bits():
    """A pair matrix of more than 2^32 bytes: the last atoms of one long graph, and the graph behind it."""
    import torch
    from paper_2506_21788_amd import binding as B
    n, d, nb = 66000, 8, 2
    off = np.array([0, n, n + 40], np.int32)
    N, G = n + 40, 2
    plan = torch.empty(B.pair_plan_workspace_bytes(N, G), dtype=torch.uint8, device="cuda")
    size = B.pair_plan(N, G, dev(off, "i32"), plan)
    assert size > 1 << 32
    pairs = torch.full((size,), B.PAIR_NONE, dtype=torch.uint8, device="cuda")
    pitch = (n + 31) // 32 * 32
    first = pairs[:n * pitch].view(n, pitch)
    first[n - 50:, n - 50:n] = 1                     # the last atoms see each other
    pairs[n * pitch:].view(40, 64)[:, :40] = 0
    gen = torch.Generator(device="cuda").manual_seed(1)
    qkv, g = torch.randn((N, 3, d), device="cuda", generator=gen), torch.randn((N, 1, d), device="cuda", generator=gen)
    bias = torch.tensor([[0.3, -0.2]], device="cuda")
    ws_b, saved_b = B.graph_attention_workspace_bytes(N, G, 1, 1, d, nb, B.F32)
    ws, saved = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    out, g_qkv, g_bias = torch.empty((N, 1, d), device="cuda"), torch.empty((N, 3, d), device="cuda"), torch.empty((1, nb), device="cuda")
    B.graph_attention_fwd(N, G, 1, 1, d, nb, B.F32, 0.35, plan, pairs, qkv, bias, out, saved)
    B.graph_attention_bwd(N, G, 1, 1, d, nb, B.F32, 0.35, plan, pairs, qkv, bias, out, saved, g, g_qkv, g_bias, ws)
    torch.cuda.synchronize()
    assert not out[:n - 50].any() and not g_qkv[:n - 50].any()
    sub = dict(off=np.array([0, 50, 90]), qkv=qkv[n - 50:].double().cpu().numpy(), g=g[n - 50:].double().cpu().numpy())
    where, p2 = ob.pair_layout(sub["off"])
    m = np.full(where[-1], 255, np.uint8)
    m[:where[1]].reshape(50, p2[0])[:, :50] = 1
    m[where[1]:].reshape(40, p2[1])[:, :40] = 0
    want = ob.graph_attention(sub["qkv"], bias.double().cpu().numpy(), m, sub["off"], 1, 1, 0.35, sub["g"])
    for a, w in zip((out[n - 50:], g_qkv[n - 50:], g_bias), want):
        assert np.allclose(a.double().cpu().numpy(), w, rtol=1e-4, atol=1e-5)


def test_more_tiles_than_one_launch_of_four_wavefronts_holds():
    """Graphs of one atom: an atom attends to itself alone, so the output is its value, D = g . v, and q and k have no gradient."""
    import torch
    from paper_2506_21788_amd import binding as B
    N, nh, nkv, d = 4_300_000, 8, 4, 8          # 4.4 million tiles; times 4 key heads and 256 threads: more than 2^32
    off = torch.arange(N + 1, dtype=torch.int32, device="cuda")
    plan = torch.empty(B.pair_plan_workspace_bytes(N, N), dtype=torch.uint8, device="cuda")
    size = B.pair_plan(N, N, off, plan)
    assert size == 32 * N
    pairs = torch.full((size,), 7, dtype=torch.uint8, device="cuda")
    pos = torch.zeros((N, 3), device="cuda")
    edge2 = torch.tensor([1.0], device="cuda")
    B.pair_buckets(N, N, plan, pos, None, None, 1, edge2, False, pairs)
    p = pairs.view(N, 32)
    assert not p[:, 0].any() and (p[:, 1:] == B.PAIR_NONE).all()
    gen = torch.Generator(device="cuda").manual_seed(2)
    qkv, g = torch.randn((N, nh + 2 * nkv, d), device="cuda", generator=gen), torch.randn((N, nh, d), device="cuda", generator=gen)
    bias = torch.zeros((nh, 2), device="cuda")
    ws_b, saved_b = B.graph_attention_workspace_bytes(N, N, nh, nkv, d, 2, B.F32)
    ws, saved = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (ws_b, saved_b))
    out, g_qkv, g_bias = torch.full_like(g, 9.0), torch.full_like(qkv, 9.0), torch.empty_like(bias)
    B.graph_attention_fwd(N, N, nh, nkv, d, 2, B.F32, 0.35, plan, pairs, qkv, bias, out, saved)
    B.graph_attention_bwd(N, N, nh, nkv, d, 2, B.F32, 0.35, plan, pairs, qkv, bias, out, saved, g, g_qkv, g_bias, ws)
    torch.cuda.synchronize()
    # the exponent c (s - m) of the only pair is formed as c s - c m, a few steps of 2^-24 of |c m| <= 64 from 0, and divides out of
    # the output again; the reverse weight 2^(c s - c m - log2 l) keeps such an error
    assert torch.allclose(out, qkv[:, nh + nkv:].repeat_interleave(2, 1), rtol=8 * 2.0 ** -24, atol=0)
    assert torch.allclose(g_qkv[:, nh + nkv:], g.view(N, nkv, 2, d).sum(2), rtol=1e-5, atol=2e-5)
    assert g_qkv[:, :nh + nkv].abs().max() < 1e-3
