"""Global attention block of a layer: every atom of a structure attends to every other one, beside the message passing between
near atoms. Owns the device buffers of one block and issues the library calls in order; no arithmetic happens here.

    y1 = norm(h; before 1)      q k v = y1 Wqkv + bqkv      a = attention(q k v; buckets, bias)      o = a Wo + bo
    z  = y1 Wg + bg (gate)      h1 = h + s1 * sigmoid(z) * norm(o; after 1)      y2 = norm(h1; before 2)
    f  = act(y2 W1 + b1)        u = f W2 + b2               h' = h1 + s2 * norm(u; after 2)
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as B


@dataclass(frozen=True)
class AttentionConfig:
    heads: int
    head_dim: int
    edges: tuple          # ascending boundaries of the distance buckets, in the unit of the positions
    ff: int               # width of the feed-forward product
    kv_heads: int | None = None     # None: one per query head
    drop_far: bool = False          # atoms beyond the last boundary do not attend to each other
    norm: str = "rms"               # or "layer"
    gate: str | None = "channel"    # "atom" or None
    act: str = "silu"               # or "gelu", "none"
    eps: float = 1e-5

    def __post_init__(self):
        # (squares are compared, and searched: a negative or falling boundary would give wrong buckets without an error)
        e = (0.0, *self.edges, float("inf"))
        assert all(a <= b for a, b in zip(e, e[1:])), f"boundaries must ascend from 0: {self.edges}"
        assert self.kv_heads is None or self.kv_heads >= 1, "kv_heads: None or at least 1"

    @property
    def kv(self):
        return self.kv_heads or self.heads

    @property
    def buckets(self):
        return len(self.edges) if self.drop_far else len(self.edges) + 1

    def fields(self, H):
        """Name -> (first value, shape) of the flat float32 parameter buffer of one block, and its length. Every field
        starts at a multiple of 8 values, so that it is 16-byte aligned in a bf16 copy too."""
        d, nh, kv = self.head_dim, self.heads, self.kv
        shapes = {"n1": (5, H), "Wqkv": (H, (nh + 2 * kv) * d), "bqkv": ((nh + 2 * kv) * d,), "bias": (nh, self.buckets),
                  "Wo": (nh * d, H), "bo": (H,)}
        if self.gate:
            zc = H if self.gate == "channel" else 1
            shapes.update(Wg=(H, zc), bg=(zc,))
        shapes.update(n2=(5, H), W1=(H, self.ff), b1=(self.ff,), W2=(self.ff, H), b2=(H,), n3=(5, H))
        out, at = {}, 0
        for k, s in shapes.items():
            out[k] = (at, s)
            n = 1
            for x in s:
                n *= x
            at += (n + 7) // 8 * 8
        return out, at


class Pairs:
    """Plan and distance buckets of a batch (one per batch, shared by all blocks)."""

    def __init__(self, cfg, N, G):
        self.cfg, self.N, self.G = cfg, N, G
        self.plan = torch.empty(max(B.pair_plan_workspace_bytes(N, G), 16), dtype=torch.uint8, device="cuda")
        self.edge2 = (torch.tensor(cfg.edges, dtype=torch.float64) ** 2).float().cuda()
        self.bytes = None

    def build(self, pos, graph_off, cell, pbc):
        """pos: the positions that the buckets are of (atoms that move between layers keep the buckets of their input positions)."""
        size = B.pair_plan(self.N, self.G, graph_off, self.plan)
        if self.bytes is None or self.bytes.numel() != size:
            self.bytes = torch.empty(size, dtype=torch.uint8, device="cuda")
        B.pair_buckets(self.N, self.G, self.plan, pos, cell, pbc, self.edge2.numel(), self.edge2, self.cfg.drop_far, self.bytes)
        return self


class AttentionBlock:
    def __init__(self, cfg, N, G, H, dtype, weights, scratch=None):
        """dtype: B.F32 or B.BF16; weights: the flat float32 device buffer of cfg.fields(H). scratch: another block of the same
        sizes on the same stream, whose workspace and gradient buffers this one shares."""
        self.cfg, self.N, self.G, self.H, self.dtype, self.W = cfg, N, G, H, dtype, weights
        self.at, n = cfg.fields(H)
        assert weights.numel() == n and weights.dtype == torch.float32, (weights.numel(), n)
        T = torch.bfloat16 if dtype == B.BF16 else torch.float32
        f32 = dict(dtype=torch.float32, device="cuda")
        t = dict(dtype=T, device="cuda")
        self.gW = torch.zeros_like(weights)          # padding between fields stays zero
        self.Wt = torch.empty(n, **t) if dtype == B.BF16 else weights
        d, nh, kv = cfg.head_dim, cfg.heads, cfg.kv
        self.cols = (nh + 2 * kv) * d
        self.norm = {"rms": B.NORM_RMS, "layer": B.NORM_LAYER}[cfg.norm]
        self.gate = {None: B.GATE_NONE, "atom": B.GATE_ATOM, "channel": B.GATE_CHANNEL}[cfg.gate]
        self.zc = {None: 0, "atom": 1, "channel": H}[cfg.gate]
        self.act = {"none": B.ACT_NONE, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}[cfg.act]
        self.scale = d ** -0.5
        F = cfg.ff
        new = lambda *s: torch.empty(s, **t)  # noqa: E731
        self.y1, self.qkv, self.a, self.o = new(N, H), new(N, nh + 2 * kv, d), new(N, nh, d), new(N, H)
        self.z = new(N, self.zc) if self.gate else None
        self.y2, self.f, self.u = new(N, H), new(N, F), new(N, H)
        self.h1 = torch.empty((N, H), **f32)
        # products: rows x inputs -> outputs
        self.shapes = {"qkv": (H, self.cols, B.ACT_NONE), "o": (nh * d, H, B.ACT_NONE), "f": (H, F, self.act), "u": (F, H, B.ACT_NONE)}
        if self.gate:
            self.shapes["z"] = (H, self.zc, B.ACT_NONE)
        size = lambda b: torch.empty(max(int(b), 16), dtype=torch.uint8, device="cuda")  # noqa: E731
        ws, self.saved = [], {}
        for k, (i, j, act) in self.shapes.items():
            w, s = B.dense_workspace_bytes(N, i, j, act, dtype)
            ws.append(w)
            self.saved[k] = size(s)
        w, s = B.graph_attention_workspace_bytes(N, G, nh, kv, d, cfg.buckets, dtype)
        ws.append(w)
        self.saved["a"] = size(s)
        w, s = B.block_norm_workspace_bytes(N, H)
        ws.append(w)
        for k in ("n1", "n2", "n3"):
            self.saved[k] = size(s)
        if scratch is not None:
            for k in ("ws", "g_wide", "g_out", "g_y", "g_z", "g_b", "g_h1"):
                setattr(self, k, getattr(scratch, k))
            return
        self.ws = size(max(ws))
        # gradients of the block's own tensors
        self.g_wide, self.g_out, self.g_y = new(N, max(self.cols, F)), new(N, nh, d), new(N, H)
        self.g_z = new(N, self.zc) if self.gate else None
        self.g_b = new(N, H)
        self.g_h1 = torch.empty((N, H), **f32)

    def _p(self, k, grad=False):
        at, s = self.at[k]
        n = 1
        for x in s:
            n *= x
        return (self.gW if grad else self.W)[at:at + n]

    def _m(self, k):
        at, s = self.at[k]
        return self.Wt[at:at + s[0] * s[1]]

    def _dense(self, k, W, b, x, y):
        i, j, act = self.shapes[k]
        B.dense_fwd(self.N, i, j, act, self.dtype, x, self._m(W), self._p(b), None, y, self.saved[k], self.ws)

    def _dense_bwd(self, k, W, b, x, g_y, g_x, r_x=None):
        i, j, act = self.shapes[k]
        B.dense_bwd(self.N, i, j, act, self.dtype, x, self._m(W), self.saved[k], g_y, g_x, self._p(W, True), self._p(b, True), self.ws,
                    r_x=r_x)

    def forward(self, pairs, h, h_out):
        """h, h_out: float32 [N,H] (may be one tensor only where no reverse pass follows)."""
        c, N, G, H = self.cfg, self.N, self.G, self.H
        if self.dtype == B.BF16:
            B.round_bf16(self.W, self.Wt)
        n = (N, H, self.norm)
        B.block_norm_fwd(*n, B.GATE_NONE, self.dtype, c.eps, h, None, None, self._p("n1"), None, self.y1, self.saved["n1"])
        self._dense("qkv", "Wqkv", "bqkv", self.y1, self.qkv)
        if self.gate:
            self._dense("z", "Wg", "bg", self.y1, self.z)
        B.graph_attention_fwd(N, G, c.heads, c.kv, c.head_dim, c.buckets, self.dtype, self.scale, pairs.plan, pairs.bytes, self.qkv,
                              self._p("bias"), self.a, self.saved["a"])
        self._dense("o", "Wo", "bo", self.a, self.o)
        B.block_norm_fwd(*n, self.gate, self.dtype, c.eps, h, self.o, self.z, self._p("n2"), self.h1, self.y2, self.saved["n2"])
        self._dense("f", "W1", "b1", self.y2, self.f)
        self._dense("u", "W2", "b2", self.f, self.u)
        B.block_norm_fwd(*n, B.GATE_NONE, self.dtype, c.eps, self.h1, self.u, None, self._p("n3"), h_out, None, self.saved["n3"])

    def backward(self, pairs, h, h_out, g_h_out, g_h):
        """g_h = gradient with respect to h; gW: of the parameters. g_h may be g_h_out."""
        c, N, G, H = self.cfg, self.N, self.G, self.H
        n = (N, H, self.norm)
        flat = self.g_wide.view(-1)
        g_f, g_qkv = flat[:N * c.ff], flat[:N * self.cols]
        B.block_norm_bwd(*n, B.GATE_NONE, self.dtype, h_out, self.u, None, self._p("n3"), self.saved["n3"], g_h_out, None, self.g_h1,
                         self.g_b, None, self._p("n3", True), self.ws)
        self._dense_bwd("u", "W2", "b2", self.f, self.g_b, g_f)
        self._dense_bwd("f", "W1", "b1", self.y2, g_f, self.g_y)
        B.block_norm_bwd(*n, self.gate, self.dtype, self.h1, self.o, self.z, self._p("n2"), self.saved["n2"], self.g_h1, self.g_y,
                         self.g_h1, self.g_b, self.g_z, self._p("n2", True), self.ws)
        self._dense_bwd("o", "Wo", "bo", self.a, self.g_b, self.g_out)
        B.graph_attention_bwd(N, G, c.heads, c.kv, c.head_dim, c.buckets, self.dtype, self.scale, pairs.plan, pairs.bytes, self.qkv,
                              self._p("bias"), self.a, self.saved["a"], self.g_out, g_qkv, self._p("bias", True), self.ws)
        if self.gate:
            self._dense_bwd("z", "Wg", "bg", self.y1, self.g_z, self.g_y)
        self._dense_bwd("qkv", "Wqkv", "bqkv", self.y1, g_qkv, self.g_y, r_x=self.g_y if self.gate else None)
        B.block_norm_bwd(*n, B.GATE_NONE, self.dtype, h, None, None, self._p("n1"), self.saved["n1"], self.g_h1, self.g_y, g_h, None, None,
                         self._p("n1", True), self.ws)
