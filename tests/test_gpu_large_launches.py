"""Calls of the attention block whose rows or values are more than one launch of 2^32 threads holds (needs a GPU)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [1, 2])
def test_block_norm_of_as_many_rows_as_it_takes(H):
    """A wavefront per row at these widths: 2^26 - 1 rows are 2^24 workgroups of 256 threads."""
    import torch
    from paper_2506_21788_amd import binding as B
    N = (1 << 26) - 1
    print("block_norm", N, H, flush=True)
    x = torch.randn((N, H), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    P = torch.tensor([1.0, 1.0, 0.0, 1.5, 0.25], device="cuda")[:, None].repeat(1, H).contiguous()
    y = torch.full((N, H), float("nan"), device="cuda")
    _, saved_b = B.block_norm_workspace_bytes(N, H)
    saved = torch.empty(saved_b, dtype=torch.uint8, device="cuda")
    B.block_norm_fwd(N, H, B.NORM_RMS, B.GATE_NONE, B.F32, 1e-5, x, None, None, P, None, y, saved)
    r = 1.0 / torch.sqrt(x.double().square().mean(1) + 1e-5)
    # a root, a quotient and a few products of float32, each half a step
    assert torch.allclose(y.double(), x.double() * r[:, None] * 1.5 + 0.25, rtol=0, atol=16 * 2.0 ** -24 * (1.5 * H + 0.25))
    assert torch.allclose(saved.view(torch.float32).view(N, 4)[:, 3].double(), r, rtol=8 * 2.0 ** -24, atol=0)
