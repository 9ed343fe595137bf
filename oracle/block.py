"""Float64 forms of the operators of a global attention block: the seam of two blocks (norms, gate, residual scale), distance
buckets of pairs, attention over the atoms of each graph with a learned bias per bucket, dense products."""
from __future__ import annotations

import itertools

import numpy as np
from scipy.special import erf

PAIR_NONE = 255


def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e)


# -- seam of two blocks -------------------------------------------------------------------------
def standardise(u, layer, eps):
    mu = u.mean(1, keepdims=True) if layer else 0.0
    r = 1.0 / np.sqrt(((u - mu) ** 2).mean(1, keepdims=True) + eps)
    return (u - mu) * r, r


def standardise_bwd(g, uh, r, layer):
    return r * (g - (g.mean(1, keepdims=True) if layer else 0.0) - uh * (g * uh).mean(1, keepdims=True))


def block_norm_fwd(x, b, z, P, layer, eps, open_next=True):
    """z: None, [N,1] or [N,H]. Returns x', y (or None)."""
    s, w1, c1, w0, c0 = P
    if b is not None:
        x = x + s * (1.0 if z is None else sigmoid(z)) * (standardise(b, layer, eps)[0] * w1 + c1)
    return x, standardise(x, layer, eps)[0] * w0 + c0 if open_next else None


def block_norm_bwd(x, b, z, P, layer, eps, g_x_out, g_y):
    """g_x, g_b, g_z, gP of block_norm_fwd; g_x_out or g_y may be None."""
    s, w1, c1, w0, _ = P
    gP = np.zeros_like(P)
    g = np.zeros_like(x) if g_x_out is None else g_x_out.copy()
    x1, _ = block_norm_fwd(x, b, z, P, layer, eps, False)
    if g_y is not None:
        xh, r = standardise(x1, layer, eps)
        gP[3], gP[4] = (g_y * xh).sum(0), g_y.sum(0)
        g = g + standardise_bwd(g_y * w0, xh, r, layer)
    if b is None:
        return g, None, None, gP
    bh, r = standardise(b, layer, eps)
    u = bh * w1 + c1
    gamma = 1.0 if z is None else sigmoid(z)
    gP[0] = (g * gamma * u).sum(0)
    q = g * s * gamma
    gP[1], gP[2] = (q * bh).sum(0), q.sum(0)
    g_z = None
    if z is not None:
        g_z = q * u * (1.0 - gamma)
        if z.shape[1] != x.shape[1] or z.shape[1] == 1:
            g_z = g_z.sum(1, keepdims=True)
    return g, standardise_bwd(q * w1, bh, r, layer), g_z, gP


# -- pairs --------------------------------------------------------------------------------------
def pair_layout(graph_off):
    """First byte of every graph's matrix (one more for the end) and the pitch of its rows."""
    n = np.diff(np.asarray(graph_off, np.int64))
    pitch = (n + 31) // 32 * 32
    return np.concatenate([[0], np.cumsum(n * pitch)]), pitch


def pair_buckets(pos, graph_off, cell, pbc, edge2, drop_far):
    """The pair matrix. float32 with every operation rounded on its own (numpy rounds each operation)."""
    f = np.float32
    pos, edge2 = np.asarray(pos, f), np.asarray(edge2, f)
    off, pitch = pair_layout(graph_off)
    out = np.full(off[-1], PAIR_NONE, np.uint8)
    for g, (a, e) in enumerate(zip(graph_off[:-1], graph_off[1:])):
        p, n = pos[a:e], int(e - a)
        best = np.full((n, n), np.inf, f)
        periodic = cell is not None and pbc is not None and bool(pbc[g])
        for s in itertools.product((-1, 0, 1), repeat=3) if periodic else [(0, 0, 0)]:
            t = np.zeros(3, f)
            if periodic:
                c = np.asarray(cell[g], f)
                t = (f(s[0]) * c[0] + f(s[1]) * c[1]) + f(s[2]) * c[2]
            r = p[:, None] - (p[None] + t)
            d2 = (r[..., 0] * r[..., 0] + r[..., 1] * r[..., 1]) + r[..., 2] * r[..., 2]
            best = np.minimum(best, d2)
        k = (best[..., None] >= edge2).sum(-1)
        k = np.where((k == len(edge2)) & bool(drop_far), PAIR_NONE, k)
        out[off[g]:off[g + 1]].reshape(n, pitch[g])[:, :n] = k
    return out


# -- attention ----------------------------------------------------------------------------------
def _graph_scores(q, k, bias, m, scale):
    """Scores [heads, i, j] of one graph, -inf where a pair is left out; k already per query head."""
    nb = bias.shape[1]
    live = m < nb
    s = np.full((q.shape[1],) + m.shape, -np.inf)
    with np.errstate(invalid="ignore"):
        raw = scale * np.einsum("ihd,jhd->hij", q, k) + bias[:, np.where(live, m, 0)]
    s[:, live] = raw[:, live]
    return s


def _graph_probs(s):
    """Softmax over j; rows without a finite score are zero."""
    top = s.max(2, keepdims=True, initial=-np.inf)
    e = np.exp(s - np.where(np.isneginf(top), 0.0, top))
    total = e.sum(2, keepdims=True)
    return e / np.where(total == 0, 1.0, total)


def graph_attention(qkv, bias, pairs, graph_off, heads, kv_heads, scale, g_out=None):
    """out [N, heads, d]; with g_out also g_qkv and g_bias. qkv [N, heads + 2 kv_heads, d]; query head h reads key and value
    head h // (heads / kv_heads). What a pair that is left out holds is not looked at."""
    off, pitch = pair_layout(graph_off)
    N, _, d = qkv.shape
    nb, rep = bias.shape[1], heads // kv_heads
    out = np.zeros((N, heads, d))
    g_qkv, g_bias = np.zeros(qkv.shape), np.zeros(bias.shape)
    for g, (a, e) in enumerate(zip(graph_off[:-1], graph_off[1:])):
        n = int(e - a)
        if n == 0:
            continue
        m = pairs[off[g]:off[g + 1]].reshape(n, pitch[g])[:, :n].astype(np.int64)
        live = m < nb
        X = qkv[a:e]
        q, k, v = X[:, :heads], np.repeat(X[:, heads:heads + kv_heads], rep, 1), np.repeat(X[:, heads + kv_heads:], rep, 1)
        p = _graph_probs(_graph_scores(q, k, bias, m, scale))
        some = live.any(0)                       # keys that somebody attends to
        v0 = np.where(some[:, None, None], v, 0.0)
        k0 = np.where(some[:, None, None], k, 0.0)
        out[a:e] = np.einsum("hij,jhd->ihd", p, v0)
        if g_out is None:
            continue
        row = live.any(1)                        # queries that attend to somebody
        go = np.where(row[:, None, None], g_out[a:e], 0.0)
        q0 = np.where(row[:, None, None], q, 0.0)
        dp = np.einsum("ihd,jhd->hij", go, v0)
        ds = p * (dp - (p * dp).sum(2, keepdims=True))
        g_qkv[a:e, :heads] = scale * np.einsum("hij,jhd->ihd", ds, k0)
        for h in range(heads):
            kh = h // rep
            g_qkv[a:e, heads + kh] += scale * ds[h].T @ q0[:, h]
            g_qkv[a:e, heads + kv_heads + kh] += p[h].T @ go[:, h]
            g_bias[h] += np.bincount(m[live], weights=ds[h][live], minlength=nb)[:nb]
    return out if g_out is None else (out, g_qkv, g_bias)


# -- dense --------------------------------------------------------------------------------------
def activation(z, act):
    """act(z) and its derivative; act: "none", "silu", "gelu"."""
    if act == "silu":
        s = sigmoid(z)
        return z * s, s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        phi = 0.5 * (1.0 + erf(z / np.sqrt(2.0)))
        return z * phi, phi + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    return z, np.ones_like(z)


def dense_fwd(x, W, b, r, act):
    z = x @ W + (0.0 if b is None else b)
    return activation(z, act)[0] + (0.0 if r is None else r)


def dense_bwd(x, W, b, act, g_y):
    g = g_y * activation(x @ W + (0.0 if b is None else b), act)[1]
    return g @ W.T, x.T @ g, g.sum(0)


# -- the whole block ----------------------------------------------------------------------------
def unpack_block(flat, fields):
    return {k: np.asarray(flat[a:a + int(np.prod(s))], np.float64).reshape(s) for k, (a, s) in fields.items()}


def attention_block_fwd(h, W, pairs, graph_off, heads, kv_heads, layer, eps, act):
    """h' and what the reverse pass needs; W: the block's parameters by name."""
    N = h.shape[0]
    d = W["Wo"].shape[0] // heads
    c = dict(h=h, W=W, pairs=pairs, off=graph_off, heads=heads, kv=kv_heads, layer=layer, eps=eps, act=act, scale=d ** -0.5)
    _, c["y1"] = block_norm_fwd(h, None, None, W["n1"], layer, eps)
    c["qkv"] = dense_fwd(c["y1"], W["Wqkv"], W["bqkv"], None, "none").reshape(N, heads + 2 * kv_heads, d)
    c["z"] = dense_fwd(c["y1"], W["Wg"], W["bg"], None, "none") if "Wg" in W else None
    c["a"] = graph_attention(c["qkv"], W["bias"], pairs, graph_off, heads, kv_heads, c["scale"]).reshape(N, heads * d)
    c["o"] = dense_fwd(c["a"], W["Wo"], W["bo"], None, "none")
    c["h1"], c["y2"] = block_norm_fwd(h, c["o"], c["z"], W["n2"], layer, eps)
    c["f"] = dense_fwd(c["y2"], W["W1"], W["b1"], None, act)
    c["u"] = dense_fwd(c["f"], W["W2"], W["b2"], None, "none")
    return block_norm_fwd(c["h1"], c["u"], None, W["n3"], layer, eps, False)[0], c


def attention_block_bwd(c, g_out):
    """Gradient with respect to h, and the parameters' by name."""
    W, layer, eps, g = c["W"], c["layer"], c["eps"], {}
    g_h1, g_u, _, g["n3"] = block_norm_bwd(c["h1"], c["u"], None, W["n3"], layer, eps, g_out, None)
    g_f, g["W2"], g["b2"] = dense_bwd(c["f"], W["W2"], W["b2"], "none", g_u)
    g_y2, g["W1"], g["b1"] = dense_bwd(c["y2"], W["W1"], W["b1"], c["act"], g_f)
    g_h, g_o, g_z, g["n2"] = block_norm_bwd(c["h"], c["o"], c["z"], W["n2"], layer, eps, g_h1, g_y2)
    g_a, g["Wo"], g["bo"] = dense_bwd(c["a"], W["Wo"], W["bo"], "none", g_o)
    N = g_a.shape[0]
    _, g_qkv, g["bias"] = graph_attention(c["qkv"], W["bias"], c["pairs"], c["off"], c["heads"], c["kv"], c["scale"],
                                          g_a.reshape(N, c["heads"], -1))
    g_y1, g["Wqkv"], g["bqkv"] = dense_bwd(c["y1"], W["Wqkv"], W["bqkv"], "none", g_qkv.reshape(N, -1))
    if g_z is not None:
        g_y, g["Wg"], g["bg"] = dense_bwd(c["y1"], W["Wg"], W["bg"], "none", g_z)
        g_y1 = g_y1 + g_y
    g_in, _, _, g["n1"] = block_norm_bwd(c["h"], None, None, W["n1"], layer, eps, g_h, g_y1)
    return g_in, g
