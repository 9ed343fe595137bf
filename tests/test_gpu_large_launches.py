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


def test_round_bf16_of_more_values_than_a_launch_has_threads_for():
    """2^35 + 9 values, 192 GiB: the launches' borders, the ends and places between."""
    import torch
    from paper_2506_21788_amd import binding as B
    n, cut = (1 << 35) + 9, ((1 << 24) - 1) * 2048
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 6 * n + (4 << 30):
        pytest.skip("needs 196 GiB of free device memory")
    print("round_bf16", n, flush=True)
    src, dst = torch.zeros(n, device="cuda"), torch.full((n,), 7.0, dtype=torch.bfloat16, device="cuda")
    try:
        where = [0, 1 << 31, (1 << 32) + 5, cut - 1100, n - 3000]
        vals = torch.randn(2200, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
        for at in where:
            src[at:at + 2200] = vals
        B.round_bf16(src, dst)
        for at in where:     # (the last two overlap)
            assert torch.equal(dst[at:at + 2200], src[at:at + 2200].to(torch.bfloat16)) and dst[at:at + 100].any(), at
        assert not dst[n - 800:].any() and not dst[1 << 30:(1 << 30) + 4096].any()
    finally:
        del src, dst
        torch.cuda.empty_cache()
