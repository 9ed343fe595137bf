"""What an attention block's configuration refuses (no GPU needed)."""
import pytest

from paper_2506_21788_amd.block import AttentionConfig


@pytest.mark.parametrize("edges", [(1.0, 3.0, 2.0), (-1.0, 2.0), (0.5, float("nan")), (float("inf"), 0.5)])
def test_boundaries_that_no_search_can_use(edges):
    with pytest.raises(AssertionError):
        AttentionConfig(heads=2, head_dim=8, edges=edges, ff=16)


def test_no_key_heads():
    with pytest.raises(AssertionError):
        AttentionConfig(heads=2, head_dim=8, edges=(1.0,), ff=16, kv_heads=0)
    assert AttentionConfig(heads=2, head_dim=8, edges=(1.0, 1.0, 2.0), ff=16).kv == 2
    assert AttentionConfig(heads=2, head_dim=8, edges=(), ff=16).buckets == 1
    assert AttentionConfig(heads=2, head_dim=8, edges=(1.0, float("inf")), ff=16, drop_far=True).buckets == 2     # all but the near ones
