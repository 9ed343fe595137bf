"""The attention block's operators run together: one block against float64, and training steps whose layers are followed by one (needs a GPU)."""
import numpy as np
import pytest

import oracle
from block_util import dev, empty
from hgnn_inputs import init_attention_weights, problem_from_batch, small_mixed_batch
from oracle import block as ob
from parity_util import TOL, assert_graph_equal, gpu_hotpath, oracle_graph, relerr

pytestmark = pytest.mark.gpu


def _config(**kw):
    from paper_2506_21788_amd.block import AttentionConfig
    return AttentionConfig(**{**dict(heads=4, head_dim=16, edges=tuple(np.linspace(0.5, 6.0, 12)), ff=96), **kw})


def _weights(cfg, H, seed):
    fields, n = cfg.fields(H)
    return init_attention_weights(np.random.default_rng(seed), H, fields, n)


def _oracle_block(cfg, H, flat):
    W = ob.unpack_block(flat, cfg.fields(H)[0])
    return lambda h, m, off: ob.attention_block_fwd(h, W, m, off, cfg.heads, cfg.kv, cfg.norm == "layer", cfg.eps, cfg.act)


def _compare_grads(name, got_flat, want, cfg, H, tol):
    scale = max(np.abs(v).max() for v in want.values())
    for k, (at, s) in cfg.fields(H)[0].items():
        a = got_flat[at:at + int(np.prod(s))].reshape(s)
        assert np.abs(a - want[k]).max() <= tol * max(np.abs(want[k]).max(), 0.05 * scale), (name, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,kw", [(64, {}), (130, dict(gate="atom", norm="layer", kv_heads=2, drop_far=True)), (256, dict(gate=None, act="gelu", heads=8, kv_heads=1)),
                                  (33, dict(head_dim=8, ff=17, act="none"))])
def test_one_block(H, kw, dtype):
    import torch
    from paper_2506_21788_amd import binding as B
    from paper_2506_21788_amd.block import AttentionBlock, Pairs
    cfg = _config(**kw)
    b = small_mixed_batch(3, n_mol=4, n_cry=4, S=2, mol_atoms=(3, 40), cry_atoms=(2, 50), cry_len=(4.0, 9.0))
    print("block", H, kw, dtype, b.N, flush=True)
    rng = np.random.default_rng(H)
    flat = _weights(cfg, H, 1)
    h, g = rng.standard_normal((b.N, H)).astype(np.float32), rng.standard_normal((b.N, H)).astype(np.float32)
    pairs = Pairs(cfg, b.N, b.G).build(dev(b.pos), dev(b.graph_off, "i32"), dev(b.cell), dev(b.pbc, "u8"))
    m = ob.pair_buckets(b.pos, b.graph_off, b.cell, b.pbc, pairs.edge2.cpu().numpy(), cfg.drop_far)
    assert np.array_equal(pairs.bytes.cpu().numpy(), m)
    blk = AttentionBlock(cfg, b.N, b.G, H, B.BF16 if dtype == "bf16" else B.F32, dev(flat))
    dh, out, g_h = dev(h), empty((b.N, H)), empty((b.N, H))
    blk.forward(pairs, dh, out)
    blk.backward(pairs, dh, out, dev(g), g_h)
    torch.cuda.synchronize()
    want, cache = _oracle_block(cfg, H, flat)(h.astype(np.float64), m, b.graph_off)
    w_h, w_W = ob.attention_block_bwd(cache, g.astype(np.float64))
    tol = TOL[dtype]
    assert relerr(out.cpu().numpy(), want) <= tol["fwd"]
    assert relerr(g_h.cpu().numpy(), w_h) <= tol["grad"]
    _compare_grads("block", blk.gW.double().cpu().numpy(), w_W, cfg, H, tol["grad"])


def _oracle_step(P, cfg, og, alpha):
    """The step of oracle.step_fwd_bwd with a block behind every layer."""
    b, hp = P["batch"], P["hp"]
    H, f = hp["H"], np.float64
    edge2 = (np.array(cfg.edges) ** 2).astype(np.float32)
    m = ob.pair_buckets(b.pos, b.graph_off, b.cell, b.pbc, edge2, cfg.drop_far)
    h, v, layers, blocks = oracle.embed_fwd(b.Z, P["emb"].astype(f)), np.zeros((b.N, 3)), [], []
    for W, Wa in zip(P["Ws"], P["Wa"]):
        h, v, c = oracle.mp_layer_fwd(h, v, og["dst"], og["col"], og["d2"].astype(f), og["rvec"].astype(f), W.astype(f), alpha)
        layers.append(c)
        h, c = _oracle_block(cfg, H, Wa)(h, m, b.graph_off)
        blocks.append(c)
    p = oracle.pool_fwd(h, b.graph_off)
    e, F, hc = oracle.heads_fwd(p, h, v, b.graph_off, b.source_id, P["Wh"].astype(f), H, hp["S"])
    g_p, g_h, g_v, _ = oracle.heads_bwd(hc, P["gE"].astype(f), P["gF"].astype(f))
    g_h = g_h + oracle.pool_bwd(g_p, b.graph_off, b.N)
    gW, gWa = [], []
    for c, cb in zip(reversed(layers), reversed(blocks)):
        g_h, ga = ob.attention_block_bwd(cb, g_h)
        g_h, g_v, gl = oracle.mp_layer_bwd(c, g_h, g_v)
        gWa.insert(0, ga)
        gW.insert(0, np.concatenate([gl[k].ravel() for k in ("W1", "b1", "W2", "b2", "wx", "W3", "b3", "W4", "b4")]))
    return e, F, gW, gWa, oracle.embed_bwd(b.Z, g_h, len(P["emb"]))


@pytest.mark.parametrize("H,dtype,kw", [(64, "f32", {}), (128, "f32", dict(gate="atom", norm="layer")), (256, "bf16", dict(heads=8, head_dim=32, kv_heads=2, ff=512))])
def test_step_with_a_block_behind_every_layer(H, dtype, kw):
    import torch
    cfg = _config(**kw)
    b = small_mixed_batch(5, n_mol=5, n_cry=4, S=3)
    P = problem_from_batch(b, 4.0, H, 2, 3, dtype, seed=2)
    P["hp"]["attn"] = cfg
    P["Wa"] = [_weights(cfg, H, 10 + l) for l in range(2)]
    hp, og = gpu_hotpath(P), oracle_graph(P)
    print("step with blocks", H, dtype, b.N, flush=True)
    gE, gF = torch.as_tensor(P["gE"]).cuda(), torch.as_tensor(P["gF"]).cuda()
    hp.build_graph()
    assert_graph_equal(hp.graph.to_numpy(), og)
    hp.step(gE, gF)
    torch.cuda.synchronize()
    e, F, gW, gWa, g_emb = _oracle_step(P, cfg, og, hp.alpha)
    tol = TOL[dtype]
    # (bf16: two layers and two blocks, each of the size of a layer)
    deep = 2.0 if dtype == "bf16" else 1.0
    assert relerr(hp.energy.cpu().numpy(), e) <= deep * tol["fwd"] and relerr(hp.force.cpu().numpy(), F) <= deep * tol["fwd"]
    for l in range(2):
        assert relerr(hp.gW[l].cpu().numpy(), gW[l]) <= deep * tol["grad"]
        _compare_grads(f"block {l}", hp.gWa[l].double().cpu().numpy(), gWa[l], cfg, H, deep * tol["grad"])
    assert relerr(hp.g_emb.cpu().numpy(), g_emb) <= deep * tol["grad"]
    # the captured step, replayed with eager steps of the same object between, gives the same bits
    want = [t.clone() for t in (hp.energy, hp.force, *hp.gW, *hp.gWa, hp.g_emb)]
    graph = hp.capture(gE, gF)
    for _ in range(3):
        for t in (hp.energy, hp.force, *hp.gW, hp.g_emb):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip((hp.energy, hp.force, *hp.gW, *hp.gWa, hp.g_emb), want))
        hp.forward()
        hp.backward(gE, gF)
        torch.cuda.synchronize()


def test_two_batches_in_turn_keep_their_own_plans():
    import torch
    cfg = _config()
    made = []
    for seed in (7, 8):
        P = problem_from_batch(small_mixed_batch(seed, S=2), 4.0, 64, 1, 2, "f32", seed=seed)
        P["hp"]["attn"], P["Wa"] = cfg, [_weights(cfg, 64, 3)]
        hp = gpu_hotpath(P)
        hp.build_graph()
        made.append((hp, torch.as_tensor(P["gE"]).cuda(), torch.as_tensor(P["gF"]).cuda()))
    first = []
    for hp, gE, gF in made:
        hp.forward()
        hp.backward(gE, gF)
        torch.cuda.synchronize()
        first.append([t.clone() for t in (hp.energy, hp.gWa[0], hp.g_emb)])
    for hp, gE, gF in made:
        hp.forward()
    for (hp, gE, gF), want in zip(made, first):
        hp.backward(gE, gF)
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip((hp.energy, hp.gWa[0], hp.g_emb), want))
