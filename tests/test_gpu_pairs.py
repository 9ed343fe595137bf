"""Pair plans and distance buckets: byte for byte against the float32 form on the host (needs a GPU)."""
import numpy as np
import pytest

from block_util import dev, room, untouched
from oracle import block as ob

pytestmark = pytest.mark.gpu


def _sizes(kind):
    return {"none": [], "one": [1], "empty ends": [0, 3, 0, 0, 33, 0], "edges": [31, 32, 33, 64, 65, 127, 1, 128],
            "many": [(7 * i) % 23 for i in range(3000)], "long": [1111]}[kind]


@pytest.mark.parametrize("kind", ["none", "one", "empty ends", "edges", "many", "long"])
@pytest.mark.parametrize("nedge,drop", [(0, False), (1, True), (31, False), (254, True)])
def test_buckets(kind, nedge, drop):
    import torch
    from paper_2506_21788_amd import binding as B
    n = np.array(_sizes(kind), np.int64)
    if kind in ("many", "long") and nedge not in (1, 31):
        pytest.skip("the small batches cover it")
    print("pair_buckets", kind, nedge, drop, flush=True)
    rng = np.random.default_rng(len(n) + nedge)
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    N, G = int(off[-1]), len(n)
    cell = (6 * np.eye(3) + 2 * rng.standard_normal((G, 3, 3)) * 0.5).astype(np.float32)
    frac = rng.random((N, 3))
    frac[::5] = np.round(frac[::5] * 2) / 2            # ties between images
    pos = np.einsum("na,nab->nb", frac, cell[np.repeat(np.arange(G), n)].astype(np.float64)).astype(np.float32)
    if N > 3:
        pos[3] = pos[1]                                # two atoms in one place
    pbc = (np.arange(G) % 2).astype(np.uint8)
    edge2 = np.sort(rng.random(nedge) * 6).astype(np.float32) ** 2
    plan = torch.empty(B.pair_plan_workspace_bytes(N, G), dtype=torch.uint8, device="cuda")
    size = B.pair_plan(N, G, dev(off, "i32"), plan)
    assert size == ob.pair_layout(off)[0][-1]
    for c, p in ((cell, pbc), (None, pbc), (cell, None)):
        got, guard = room(size)
        B.pair_buckets(N, G, plan, dev(pos), dev(c), dev(p, "u8"), nedge, dev(edge2), drop, got)
        assert np.array_equal(got.cpu().numpy(), ob.pair_buckets(pos, off, c, p, edge2, drop)) and untouched(guard)


@pytest.mark.parametrize("drop", [False, True])
@pytest.mark.parametrize("tall", [12.03, 12.1, 30.0])
def test_cells_more_than_twice_as_high_as_the_last_boundary(tall, drop):
    """Where one image per pair is looked at: heights just above (and below) twice the last boundary, ties between images, atoms on the
    faces, outside the cell and far away, pairs at a boundary's very distance."""
    import torch
    from paper_2506_21788_amd import binding as B
    rng = np.random.default_rng(int(tall * 10))
    edge = np.array([1.0, 2.5, 4.0, 6.0], np.float32)
    cells = np.stack([np.diag([tall, tall, tall]), np.diag([tall, 40.0, 17.0]), tall * np.eye(3) + np.tril(rng.random((3, 3)) * 4, -1),
                      np.diag([11.9, 30.0, 30.0]), tall * np.eye(3)[[1, 2, 0]]]).astype(np.float32)
    n = np.array([150, 97, 200, 64, 33])
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    N, G = int(off[-1]), len(n)
    frac = rng.random((N, 3))
    frac[::4] = np.round(frac[::4] * 4) / 4
    frac[5] += 1.0                                   # outside the cell by one, by three, and far away
    frac[6] -= 3.0
    pos = np.einsum("na,nab->nb", frac, cells[np.repeat(np.arange(G), n)].astype(np.float64)).astype(np.float32)
    pos[7] += 2.0e4
    pos[10] = pos[9] + np.array([6.0, 0, 0], np.float32)
    pos[12] = pos[11] + np.array([0, 5.9999995, 0], np.float32)
    pos[14] = np.nan
    plan = torch.empty(B.pair_plan_workspace_bytes(N, G), dtype=torch.uint8, device="cuda")
    got, guard = room(B.pair_plan(N, G, dev(off, "i32"), plan))
    B.pair_buckets(N, G, plan, dev(pos), dev(cells), dev(np.ones(G), "u8"), 4, dev(edge ** 2), drop, got)
    want = ob.pair_buckets(np.where(np.isnan(pos), np.float32(1e18), pos), off, cells, np.ones(G), edge ** 2, drop)
    assert untouched(guard)
    where, pitch = ob.pair_layout(off)
    m = want[:where[1]].reshape(150, pitch[0])
    beyond = 255 if drop else 4
    m[14, :150] = m[:, 14] = beyond                  # (also to itself)
    assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("n", [200, 257, 1031, 1300])
@pytest.mark.parametrize("shape", ["cube", "oblique", "long"])
def test_roomy_cells_of_many_columns(shape, n):
    """Several runs of 256 columns of a roomy cell, the last one cut; oblique cells and ones 15 times as long as high; pairs on the
    boundary between two images; atoms whose fractional coordinates are not to be trusted among the others."""
    import torch
    from paper_2506_21788_amd import binding as B
    rng = np.random.default_rng(n + len(shape))
    edge = np.array([0.5, 1.0, 1.7, 2.0], np.float32)
    cell = {"cube": 9.0 * np.eye(3), "oblique": np.array([[9.0, 0, 0], [7.0, 6, 0], [-5, 4, 6]]), "long": np.array([[60.0, 0, 0], [11, 4.6, 0], [-20, 1.5, 4.7]])}[shape]
    frac = rng.random((n, 3))
    frac[::3] = np.round(frac[::3] * 2) / 2
    frac[1::7] += rng.integers(-1, 2, (len(frac[1::7]), 3))
    pos = (frac @ cell).astype(np.float32)
    pos[n // 2] += 250.0                               # more than 100 boundaries away
    pos[n - 1] -= 1.0e6
    pos[3] = pos[5]
    off = np.array([0, n], np.int32)
    plan = torch.empty(B.pair_plan_workspace_bytes(n, 1), dtype=torch.uint8, device="cuda")
    size = B.pair_plan(n, 1, dev(off, "i32"), plan)
    cell = cell.astype(np.float32)[None]
    for drop in (False, True):
        got, guard = room(size)
        B.pair_buckets(n, 1, plan, dev(pos), dev(cell), dev(np.ones(1), "u8"), 4, dev(edge ** 2), drop, got)
        want = ob.pair_buckets(pos, off, cell, np.ones(1), edge ** 2, drop)
        assert np.array_equal(got.cpu().numpy(), want) and untouched(guard)
        assert (want < (4 if not drop else 255)).sum() > 2 * n     # (there is something to find)


def test_distance_that_is_no_number_is_beyond_every_boundary():
    import torch
    from paper_2506_21788_amd import binding as B
    pos = torch.tensor([[0.0, 0, 0], [float("nan"), 0, 0], [float("inf"), 0, 0]], device="cuda")
    plan = torch.empty(B.pair_plan_workspace_bytes(3, 1), dtype=torch.uint8, device="cuda")
    m = torch.empty(B.pair_plan(3, 1, dev(np.array([0, 3]), "i32"), plan), dtype=torch.uint8, device="cuda")
    B.pair_buckets(3, 1, plan, pos, None, None, 2, dev(np.array([1.0, 4.0])), False, m)
    assert m.view(3, 32)[:, :3].tolist() == [[0, 2, 2], [2, 2, 2], [2, 2, 2]]


@pytest.mark.parametrize("off", [[1, 5], [0, 4], [0, 6], [0, 3, 2, 5], [0, -1, 5], [0, 9, 5]])
def test_bad_offsets_are_found_and_leave_an_empty_plan(off):
    import torch
    from paper_2506_21788_amd import binding as B
    N, G = 5, len(off) - 1
    plan = torch.empty(B.pair_plan_workspace_bytes(N, G), dtype=torch.uint8, device="cuda")
    with pytest.raises(B.HgnnError) as e:
        B.pair_plan(N, G, dev(np.array(off), "i32"), plan)
    assert e.value.code == -3
    m = torch.full((512,), 7, dtype=torch.uint8, device="cuda")
    B.pair_buckets(N, G, plan, torch.zeros((N, 3), device="cuda"), None, None, 1, torch.ones(1, device="cuda"), False, m)
    assert bool((m == 7).all())
