"""Refusals of the attention block's entry points: found on the host, before any launch (no GPU needed)."""
import ctypes
import os

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2506_21788_amd", "libhgnn.so")
NULL, SHAPE, WS, OVERFLOW = -1, -2, -6, -7
i32, i64, f32, vp, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
P = vp(0x1000)      # never dereferenced


def _lib():
    lib = ctypes.CDLL(LIB)
    lib.hgnn_last_error_string.restype = ctypes.c_char_p
    return lib


def test_block_norm():
    lib = _lib()
    a, b = sz(0), sz(0)
    size = lambda N, H: lib.hgnn_block_norm_workspace_bytes(i32(N), i32(H), ctypes.byref(a), ctypes.byref(b))  # noqa: E731
    assert size(10, 1024) == 0 and b.value == 160 and size(0, 1) == 0
    assert size(10, 1025) == SHAPE and size(10, 0) == SHAPE and size(-1, 4) == SHAPE
    assert lib.hgnn_block_norm_workspace_bytes(i32(1), i32(1), None, ctypes.byref(b)) == NULL

    def fwd(N=4, H=8, norm=0, gate=0, dt=0, eps=1e-5, x=P, blk=P, z=None, par=P, xo=P, y=P, saved=None, sb=0):
        return lib.hgnn_block_norm_fwd(None, i32(N), i32(H), i32(norm), i32(gate), i32(dt), f32(eps), x, blk, z, par, xo, y, saved, sz(sb))
    for kw, code in ((dict(norm=2), SHAPE), (dict(gate=3), SHAPE), (dict(dt=2), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
                     (dict(blk=None, gate=1, z=P), SHAPE), (dict(gate=2), NULL), (dict(x=None), NULL), (dict(par=None), NULL),
                     (dict(xo=None), NULL), (dict(blk=None, y=None), NULL), (dict(saved=P, sb=63), WS), (dict(N=0, x=None), 0)):
        assert fwd(**kw) == code, kw

    def bwd(N=4, H=8, gate=0, xo=P, blk=P, z=None, saved=P, sb=64, gxo=P, gy=P, gx=P, gb=P, gz=None, gP=P, ws=P, wb=1 << 20):
        return lib.hgnn_block_norm_bwd(None, i32(N), i32(H), i32(0), i32(gate), i32(0), xo, blk, z, P, saved, sz(sb), gxo, gy, gx, gb, gz, gP,
                                       ws, sz(wb))
    for kw, code in ((dict(wb=8), WS), (dict(sb=63), WS), (dict(gP=None), NULL), (dict(gxo=None, gy=None), NULL), (dict(xo=None), NULL),
                     (dict(gb=None), NULL), (dict(gate=1, z=P), NULL), (dict(gate=1, gz=P), NULL), (dict(saved=None), NULL), (dict(H=2000), SHAPE)):
        assert bwd(**kw) == code, kw


def test_pairs():
    lib = _lib()
    a = sz(0)
    size = lambda N, G: lib.hgnn_pair_plan_workspace_bytes(i32(N), i32(G), ctypes.byref(a))  # noqa: E731
    assert size(0, 0) == 0 and size(1000, 10) == 0 and a.value > 12 * 11
    assert size(-1, 1) == SHAPE and size(1, -1) == SHAPE and size(1 << 28, 1) == OVERFLOW and size(1, 1 << 28) == OVERFLOW
    out = i64(0)
    plan = lambda off=P, p=P, pb=1 << 20, o=ctypes.byref(out): lib.hgnn_pair_plan(None, i32(5), i32(1), off, p, sz(pb), o)  # noqa: E731
    assert plan(off=None) == NULL and plan(p=None) == NULL and plan(o=None) == NULL and plan(pb=8) == WS

    def buckets(N=5, p=P, pb=1 << 20, pos=P, ne=3, e=P, m=P):
        return lib.hgnn_pair_buckets(None, i32(N), i32(1), p, sz(pb), pos, None, None, i32(ne), e, i32(0), m)
    for kw, code in ((dict(ne=-1), SHAPE), (dict(ne=255), SHAPE), (dict(p=None), NULL), (dict(pos=None), NULL), (dict(e=None), NULL),
                     (dict(m=None), NULL), (dict(pb=8), WS), (dict(N=-1), SHAPE), (dict(N=0, pos=None), 0)):
        assert buckets(**kw) == code, kw


def test_graph_attention():
    lib = _lib()
    a, b = sz(0), sz(0)

    def size(N=100, G=3, nh=4, kv=2, d=32, nb=8, dt=0):
        return lib.hgnn_graph_attention_workspace_bytes(i32(N), i32(G), i32(nh), i32(kv), i32(d), i32(nb), i32(dt), ctypes.byref(a), ctypes.byref(b))
    assert size() == 0 and b.value >= 4 * 100 * 4 and size(dt=1) == 0 and b.value >= 4 * 100 * 4 + 4 * 100 * 4 * 32
    for kw, code in ((dict(N=-1), SHAPE), (dict(G=-1), SHAPE), (dict(nh=0), SHAPE), (dict(nh=65, kv=1), SHAPE), (dict(kv=3), SHAPE), (dict(kv=0), SHAPE),
                     (dict(kv=8), SHAPE), (dict(d=4), SHAPE), (dict(d=12), SHAPE), (dict(d=136), SHAPE), (dict(nb=0), SHAPE), (dict(nb=65), SHAPE),
                     (dict(dt=2), SHAPE), (dict(N=1 << 28), OVERFLOW), (dict(N=200_000_000, G=100_000_000, nh=64, kv=1), OVERFLOW)):
        assert size(**kw) == code, kw

    def fwd(N=100, plan=P, pb=1 << 20, pairs=P, qkv=P, bias=P, out=P, saved=None, sb=0, scale=1.0):
        return lib.hgnn_graph_attention_fwd(None, i32(N), i32(3), i32(4), i32(2), i32(32), i32(8), i32(0), f32(scale), plan, sz(pb), pairs, qkv, bias,
                                            out, saved, sz(sb))
    for kw, code in ((dict(plan=None), NULL), (dict(pairs=None), NULL), (dict(qkv=None), NULL), (dict(bias=None), NULL), (dict(out=None), NULL),
                     (dict(pb=64), WS), (dict(saved=P, sb=64), WS), (dict(N=0, qkv=None), 0), (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE),
                     (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE)):
        assert fwd(**kw) == code, kw

    def bwd(pb=1 << 20, saved=P, sb=1 << 20, g=P, gq=P, gb=P, ws=P, wb=1 << 20, out=P):
        return lib.hgnn_graph_attention_bwd(None, i32(100), i32(3), i32(4), i32(2), i32(32), i32(8), i32(0), f32(1.0), P, sz(pb), P, P, P, out, saved,
                                            sz(sb), g, gq, gb, ws, sz(wb))
    for kw, code in ((dict(pb=64), WS), (dict(sb=64), WS), (dict(wb=64), WS), (dict(saved=None), NULL), (dict(g=None), NULL), (dict(gq=None), NULL),
                     (dict(gb=None), NULL), (dict(ws=None), NULL), (dict(out=None), NULL)):
        assert bwd(**kw) == code, kw


def test_dense():
    lib = _lib()
    a, b = sz(0), sz(0)

    def size(M=4000, K=64, N=96, act=1, dt=0):
        return lib.hgnn_dense_workspace_bytes(i32(M), i32(K), i32(N), i32(act), i32(dt), ctypes.byref(a), ctypes.byref(b))
    assert size() == 0 and b.value == 4000 * 96 * 4 and a.value > 0
    assert size(act=0) == 0 and b.value == 0 and size(M=0) == 0 and a.value == 0
    for kw, code in ((dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(N=0), SHAPE), (dict(K=8193), SHAPE), (dict(N=8193), SHAPE), (dict(act=3), SHAPE),
                     (dict(dt=2), SHAPE), (dict(M=(1 << 26) + 1), OVERFLOW)):
        assert size(**kw) == code, kw
    fwd = lambda x=P, W=P, y=P, s=None, sb=0, M=40, ws=P, wb=1 << 30: lib.hgnn_dense_fwd(None, i32(M), i32(64), i32(96), i32(1), i32(0), x, W, None, None, y, s, sz(sb), ws, sz(wb))  # noqa: E731
    for kw, code in ((dict(x=None), NULL), (dict(W=None), NULL), (dict(y=None), NULL), (dict(s=P, sb=8), WS), (dict(M=0, x=None), 0),
                     (dict(M=40000, ws=None), NULL), (dict(M=40000, wb=8), WS)):
        assert fwd(**kw) == code, kw

    def bwd(x=P, W=P, s=P, sb=1 << 30, g=P, gx=P, gW=P, ws=P, wb=1 << 30, M=4000):
        return lib.hgnn_dense_bwd(None, i32(M), i32(64), i32(96), i32(1), i32(0), x, W, s, sz(sb), g, P, gx, gW, P, ws, sz(wb))
    for kw, code in ((dict(x=None), NULL), (dict(gx=None), NULL), (dict(W=None), NULL), (dict(s=None), NULL), (dict(g=None), NULL), (dict(gW=None), NULL), (dict(ws=None), NULL),
                     (dict(wb=8), WS), (dict(sb=8), WS)):
        assert bwd(**kw) == code, kw
    assert lib.hgnn_round_bf16(None, i64(-1), P, P) == SHAPE and lib.hgnn_round_bf16(None, i64(4), None, P) == NULL
    assert lib.hgnn_round_bf16(None, i64(1 << 42), P, P) == OVERFLOW and lib.hgnn_round_bf16(None, i64(0), None, None) == 0


def test_more_rows_and_tiles_than_a_launch_can_hold():
    lib = _lib()
    a, b = sz(0), sz(0)
    norm = lambda N: lib.hgnn_block_norm_workspace_bytes(i32(N), i32(8), ctypes.byref(a), ctypes.byref(b))  # noqa: E731
    assert norm((1 << 26) - 1) == 0 and norm(1 << 26) == OVERFLOW
    assert lib.hgnn_block_norm_fwd(None, i32(1 << 26), i32(8), i32(0), i32(0), i32(0), f32(1e-5), P, P, None, P, P, P, None, sz(0)) == OVERFLOW
    # 2^22 graphs of one atom: 2^22 + 2^17 tiles, 2^32 threads and more with 16 heads and a wavefront each
    att = lambda nh: lib.hgnn_graph_attention_workspace_bytes(i32(1 << 22), i32(1 << 22), i32(nh), i32(1), i32(8), i32(1), i32(0), ctypes.byref(a),  # noqa: E731
                                                              ctypes.byref(b))
    assert att(15) == 0 and att(16) == OVERFLOW
