"""Pins of the float64 forms of the attention block's operators: central differences, closed forms, invariances (CPU)."""
import numpy as np
import pytest

from oracle import block as ob


def _differences(f, x, n, rng, h=1e-6):
    """(places, central differences of the scalar f at n random places of x); x is changed in place and restored."""
    flat = x.reshape(-1)
    at = rng.choice(flat.size, min(n, flat.size), replace=False)
    out = []
    for i in at:
        keep = flat[i]
        flat[i] = keep + h
        up = f()
        flat[i] = keep - h
        down = f()
        flat[i] = keep
        out.append((up - down) / (2 * h))
    return at, np.array(out)


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", [None, "atom", "channel"])
def test_block_norm_gradients_by_differences(layer, gate):
    rng = np.random.default_rng(1)
    N, H = 5, 7
    x, b = rng.standard_normal((N, H)), rng.standard_normal((N, H))
    z = None if gate is None else rng.standard_normal((N, 1 if gate == "atom" else H))
    P = rng.standard_normal((5, H))
    gx, gy = rng.standard_normal((N, H)), rng.standard_normal((N, H))

    def loss():
        x1, y = ob.block_norm_fwd(x, b, z, P, layer, 1e-5)
        return (x1 * gx).sum() + (y * gy).sum()

    g_x, g_b, g_z, gP = ob.block_norm_bwd(x, b, z, P, layer, 1e-5, gx, gy)
    for v, g in ((x, g_x), (b, g_b), (z, g_z), (P, gP)):
        if v is not None:
            at, d = _differences(loss, v, 20, rng)
            assert np.allclose(g.reshape(-1)[at], d, rtol=1e-6, atol=1e-7)


def test_block_norm_of_a_constant_row_is_finite():
    P = np.ones((5, 4))
    _, y = ob.block_norm_fwd(np.full((1, 4), 3.0), None, None, P, True, 1e-5)
    assert np.allclose(y, 1.0)          # the shift alone
    assert np.isfinite(ob.block_norm_bwd(np.zeros((1, 4)), None, None, P, False, 1e-5, None, np.ones((1, 4)))[0]).all()


@pytest.mark.parametrize("heads,kv", [(3, 3), (4, 2), (4, 1)])
def test_attention_gradients_by_differences(heads, kv):
    rng = np.random.default_rng(2)
    off = np.array([0, 4, 4, 5, 11])
    N, d, nb = 11, 3, 4
    qkv, bias = rng.standard_normal((N, heads + 2 * kv, d)), rng.standard_normal((heads, nb))
    size = ob.pair_layout(off)[0][-1]
    pairs = rng.integers(0, nb + 2, size).astype(np.uint8)
    g = rng.standard_normal((N, heads, d))
    loss = lambda: (ob.graph_attention(qkv, bias, pairs, off, heads, kv, 0.7) * g).sum()  # noqa: E731
    _, g_qkv, g_bias = ob.graph_attention(qkv, bias, pairs, off, heads, kv, 0.7, g)
    for v, gv in ((qkv, g_qkv), (bias, g_bias)):
        at, diff = _differences(loss, v, 40, rng)
        assert np.allclose(gv.reshape(-1)[at], diff, rtol=1e-6, atol=1e-7)


def test_attention_of_equal_scores_is_the_mean_and_empty_rows_are_zero():
    off = np.array([0, 3])
    qkv = np.zeros((3, 3, 2))
    qkv[:, 2] = [[1, 2], [3, 4], [5, 6]]
    pairs = np.full((3, 32), ob.PAIR_NONE, np.uint8)
    pairs[0, :3] = 0
    pairs[1, 1] = 0
    out = ob.graph_attention(qkv, np.zeros((1, 1)), pairs.reshape(-1), off, 1, 1, 1.0)
    assert np.allclose(out[:, 0], [[3, 4], [3, 4], [0, 0]])


def test_attention_does_not_look_at_what_nobody_attends_to():
    rng = np.random.default_rng(3)
    off = np.array([0, 4])
    qkv, bias = rng.standard_normal((4, 3, 2)), np.zeros((1, 2))
    pairs = np.full((4, 32), 1, np.uint8)
    pairs[2] = pairs[:, 2] = ob.PAIR_NONE
    want = ob.graph_attention(qkv, bias, pairs.reshape(-1), off, 1, 1, 1.0, np.ones((4, 1, 2)))
    qkv[2] = np.nan
    got = ob.graph_attention(qkv, bias, pairs.reshape(-1), off, 1, 1, 1.0, np.ones((4, 1, 2)))
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


def test_buckets_against_distances_in_float64_and_images():
    rng = np.random.default_rng(4)
    off = np.array([0, 5, 12])
    cell = np.stack([np.diag([9.0, 10.0, 11.0])] * 2)
    pos = rng.random((12, 3)) * [9.0, 10.0, 11.0]
    edge = np.array([1.0, 2.0, 4.0])
    m = ob.pair_buckets(pos, off, cell, [0, 1], edge ** 2, True)
    o, pitch = ob.pair_layout(off)
    assert list(pitch) == [32, 32] and m.size == 12 * 32
    for g, (a, e) in enumerate(zip(off[:-1], off[1:])):
        r = pos[a:e][:, None] - pos[a:e][None]
        if g == 1:
            r -= np.round(r / np.diag(cell[1])) * np.diag(cell[1])     # nearest image of an orthogonal cell
        want = (np.linalg.norm(r, axis=2)[..., None] >= edge).sum(-1)
        got = m[o[g]:o[g + 1]].reshape(e - a, 32)
        assert np.array_equal(got[:, :e - a], np.where(want == 3, 255, want)) and (got[:, e - a:] == 255).all()


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_dense_gradients_by_differences(act):
    rng = np.random.default_rng(5)
    x, W, b, g = rng.standard_normal((4, 3)), rng.standard_normal((3, 5)), rng.standard_normal(5), rng.standard_normal((4, 5))
    loss = lambda: (ob.dense_fwd(x, W, b, None, act) * g).sum()  # noqa: E731
    for v, gv in zip((x, W, b), ob.dense_bwd(x, W, b, act, g)):
        at, d = _differences(loss, v, 15, rng)
        assert np.allclose(gv.reshape(-1)[at], d, rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("gate", [None, "atom", "channel"])
def test_block_gradients_by_differences(gate):
    rng = np.random.default_rng(6)
    off, H, nh, kv, d, F, nb = np.array([0, 3, 8]), 6, 2, 1, 4, 5, 3
    shapes = {"n1": (5, H), "Wqkv": (H, (nh + 2 * kv) * d), "bqkv": ((nh + 2 * kv) * d,), "bias": (nh, nb), "Wo": (nh * d, H), "bo": (H,),
              "n2": (5, H), "W1": (H, F), "b1": (F,), "W2": (F, H), "b2": (H,), "n3": (5, H)}
    if gate:
        shapes.update(Wg=(H, 1 if gate == "atom" else H), bg=(1 if gate == "atom" else H,))
    W = {k: 0.5 * rng.standard_normal(s) for k, s in shapes.items()}
    pairs = rng.integers(0, nb + 1, ob.pair_layout(off)[0][-1]).astype(np.uint8)
    h, g = rng.standard_normal((8, H)), rng.standard_normal((8, H))
    run = lambda: ob.attention_block_fwd(h, W, pairs, off, nh, kv, gate == "atom", 1e-5, "silu")  # noqa: E731
    g_h, gW = ob.attention_block_bwd(run()[1], g)
    loss = lambda: (run()[0] * g).sum()  # noqa: E731
    for v, gv in [(h, g_h)] + [(W[k], gW[k]) for k in shapes]:
        at, diff = _differences(loss, v, 12, rng)
        assert np.allclose(gv.reshape(-1)[at], diff, rtol=1e-5, atol=1e-7)
