"""Training steps with attention blocks behind layers of the other kinds (radial basis, moving atoms, position gradients), and replays that
have to write every gradient (needs a GPU)."""
import numpy as np
import pytest

import oracle
from hgnn_inputs import small_mixed_batch
from oracle import block as ob
from parity_util import TOL, gpu_hotpath, oracle_graph, problem_from_batch, relerr
from test_gpu_attention_block import _compare_grads, _config, _oracle_block, _weights

pytestmark = pytest.mark.gpu


def _problem(H, dtype, seed, cfg, **hp):
    P = problem_from_batch(small_mixed_batch(seed, n_mol=4, n_cry=3, S=2), 4.0, H, 2, 2, dtype, seed=seed, **hp)
    P["hp"]["attn"] = cfg
    P["Wa"] = [_weights(cfg, H, 20 + l) for l in range(2)]
    return P


def _oracle_step(P, cfg, og, alpha):
    """oracle.step_fwd_bwd with a block behind every layer: the blocks' buckets are those of the input positions and have no gradient."""
    b, hp, f = P["batch"], P["hp"], np.float64
    H, move, grad = hp["H"], hp.get("move", False), hp.get("pos_grad", False) or hp.get("move", False)
    rbf = hp.get("rbf_k")
    m = ob.pair_buckets(b.pos, b.graph_off, b.cell, b.pbc, (np.array(cfg.edges) ** 2).astype(np.float32), cfg.drop_far)
    h, v, layers, blocks, geom = oracle.embed_fwd(b.Z, P["emb"].astype(f)), np.zeros((b.N, 3)), [], [], []
    for W, Wa in zip(P["Ws"], P["Wa"]):
        r, d2 = og["rvec"].astype(f), og["d2"].astype(f)
        if move:
            r, d2 = oracle.edge_geometry(og["rvec"], v, og["dst"], og["col"])
        attr = oracle.edge_rbf(d2, rbf, hp["rc"]) if rbf else None
        h, v, c = oracle.mp_layer_fwd(h, v, og["dst"], og["col"], d2, r, W.astype(f), alpha, attr=attr)
        layers.append(c)
        geom.append((r, d2))
        h, c = _oracle_block(cfg, H, Wa)(h, m, b.graph_off)
        blocks.append(c)
    p = oracle.pool_fwd(h, b.graph_off)
    e, F, hc = oracle.heads_fwd(p, h, v, b.graph_off, b.source_id, P["Wh"].astype(f), H, hp["S"])
    g_p, g_h, g_v, _ = oracle.heads_bwd(hc, P["gE"].astype(f), P["gF"].astype(f))
    g_h = g_h + oracle.pool_bwd(g_p, b.graph_off, b.N)
    gW, gWa, g_r0 = [], [], np.zeros((len(og["dst"]), 3))
    for c, cb, (r, d2) in zip(reversed(layers), reversed(blocks), reversed(geom)):
        g_h, ga = ob.attention_block_bwd(cb, g_h)
        g_h, g_v, gl, g_attr, g_rvec = oracle.mp_layer_bwd(c, g_h, g_v, edge_grads=True)
        if grad:
            g_d2 = oracle.edge_rbf_bwd(d2, rbf, hp["rc"], g_attr) if rbf else g_attr[:, 0]
            g_r, g_vg = oracle.edge_geometry_bwd(r, g_rvec, g_d2, og["dst"], og["col"], b.N)
            g_r0 += g_r
            g_v = g_v + g_vg if move else g_v
        gWa.insert(0, ga)
        gW.insert(0, np.concatenate([gl[k].ravel() for k in ("W1", "b1", "W2", "b2", "wx", "W3", "b3", "W4", "b4")]))
    g_pos = np.zeros((b.N, 3))
    np.add.at(g_pos, og["dst"], g_r0)
    np.add.at(g_pos, og["col"], -g_r0)
    return e, F, gW, gWa, oracle.embed_bwd(b.Z, g_h, len(P["emb"])), g_pos


@pytest.mark.parametrize("H,dtype,hp", [(64, "bf16", dict(rbf_k=8)), (128, "bf16", dict(rbf_k=6, pos_grad=True)), (64, "f32", dict(pos_grad=True)),
                                        (64, "f32", dict(move=True)), (128, "bf16", dict(rbf_k=5, move=True, pos_grad=True))])
def test_layers_of_every_kind(H, dtype, hp):
    import torch
    cfg = _config(head_dim=8, gate="atom")
    P = _problem(H, dtype, 31, cfg, **hp)
    print("step with blocks", H, dtype, hp, flush=True)
    path, og = gpu_hotpath(P), oracle_graph(P)
    path.build_graph()
    path.step(torch.as_tensor(P["gE"]).cuda(), torch.as_tensor(P["gF"]).cuda())
    torch.cuda.synchronize()
    e, F, gW, gWa, g_emb, g_pos = _oracle_step(P, cfg, og, path.alpha)
    # (two layers, and two blocks of the size of a layer)
    tol = {k: 2.0 * v for k, v in TOL[dtype].items()}
    assert relerr(path.energy.cpu().numpy(), e) <= tol["fwd"] and relerr(path.force.cpu().numpy(), F) <= tol["fwd"]
    for l in range(2):
        assert relerr(path.gW[l].cpu().numpy(), gW[l]) <= tol["grad"]
        _compare_grads(f"block {l}", path.gWa[l].double().cpu().numpy(), gWa[l], cfg, H, tol["grad"])
    assert relerr(path.g_emb.cpu().numpy(), g_emb) <= tol["grad"]
    if hp.get("pos_grad") or hp.get("move"):
        assert relerr(path.g_pos.cpu().numpy(), g_pos) <= tol["grad"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_replays_write_every_gradient_of_the_blocks(dtype):
    import torch
    H, cfg = 64, _config()
    P = _problem(H, dtype, 33, cfg)
    path = gpu_hotpath(P)
    gE, gF = torch.as_tensor(P["gE"]).cuda(), torch.as_tensor(P["gF"]).cuda()
    path.build_graph()
    path.step(gE, gF)
    torch.cuda.synchronize()
    fields, _ = cfg.fields(H)
    views = [w[at:at + int(np.prod(s))] for w in path.gWa for at, s in fields.values()]      # all but the padding
    want = [v.clone() for v in views]
    graph = path.capture(gE, gF)
    for _ in range(3):
        for v in views:
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, w) for v, w in zip(views, want))
        path.forward()
        path.backward(gE, gF)
        torch.cuda.synchronize()


def test_profile_shows_the_blocks_by_class():
    """One launch scope per call: of a step with two gated blocks 6 norms each, 2 attention calls, 10 dense products and a copy of the weights."""
    import torch
    from paper_2506_21788_amd import binding as B
    P = _problem(64, "bf16", 35, _config())
    path = gpu_hotpath(P)
    gE, gF = torch.as_tensor(P["gE"]).cuda(), torch.as_tensor(P["gF"]).cuda()

    def count(work):
        torch.cuda.synchronize()
        B.profile_begin((1 << B.profile_num_tags()) - 1)
        work()
        B.profile_end()
        return {B.profile_tag_name(t): B.profile_read(t) for t in range(B.profile_num_tags())}

    got = count(path.build_graph)
    assert got["pairs"][0] == 2 and got["pairs"][1] > 0.0
    path.step(gE, gF)
    got = count(lambda: (path.forward(), path.backward(gE, gF)))
    assert [got[k][0] for k in ("block_norm", "attention", "dense", "pairs")] == [12, 4, 22, 0]
    assert all(got[k][1] > 0.0 for k in ("block_norm", "attention", "dense"))
